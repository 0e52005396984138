// Packed-token linear operator on 8-bit rows:
//   y = act(x_scale w_scale (x w^T) + bias) + residual
// with x int8 [T, K], w int8 [N, K], the products summed exactly in int32 on the matrix
// cores (v_mfma_i32_16x16x64_i8; K <= 131056 keeps the sums below 2^31) and scales, bias, activation and
// residual applied in fp32 to the finished sum, which is rounded to the type once.
//
// A TM x TN tile per workgroup of WM x WN (x WK, over k) waves.  Operands go global -> LDS
// by bounds-checked direct copies, 128 k (one 128-byte line) of each row per stage, ST stages; the
// 16-byte chunks of a row are XOR-swizzled by it, so fragment reads of 16 rows meet distinct
// bank groups.  Rows past T or N lie outside the descriptors, chunks past K are sent past
// them: both arrive as zeros.
// A lane's fragment is 16 consecutive k of one row in both operands, and the tile is
// computed as w x^T, so that a lane ends with four consecutive features of one token.
#include <type_traits>

#include "gemm_common.h"

namespace rag {
namespace {

typedef __attribute__((ext_vector_type(4))) int intx4;

template <int TM_, int TN_, int WM_, int WN_, int WK_, int ST_>
struct I8Cfg {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, WK = WK_, ST = ST_;
    static constexpr int kWaves = WM * WN * WK, kThreads = kWave * kWaves;
    static constexpr int FM = TM / WM / 16, FN = TN / WN / 16;  // 16-wide blocks of a wave
    static constexpr int kStage = (TM + TN) * 128;              // bytes
    static constexpr int kCopies = (TM + TN) / 8 / kWaves;      // 1 KB copies per wave and stage
    static constexpr int G = 2 / WK;                            // 64-k groups per wave and stage
    static constexpr int kRows = 65536 / (TN * WK * 4) < TM ? 65536 / (TN * WK * 4) : TM;  // epilogue slice
    static constexpr int kSum = kRows * TN * WK * 4;
    static constexpr int kLds = ST * kStage > kSum ? ST * kStage : kSum;
    static_assert((TM + TN) / 8 % kWaves == 0 && kLds <= 160 * 1024 && (WK == 1 || WK == 2), "configuration");
    static_assert(TM / WM % 16 == 0 && TN / WN % 16 == 0 && TM % kRows == 0 && (TM / WM) % 16 == 0, "blocks");
};

struct I8Args {
    const int8_t* x;
    const float* x_scale;
    const int8_t* w;
    const float* w_scale;
    const void* bias;
    const void* residual;
    void* y;
    int ldx, ldr, ldy, T, K, N;
};

constexpr int kPast = 0x7ffffff0;  // a byte offset past every descriptor: reads as zero

// LDS wait and barrier the compiler's own wait insertion sees, so that it adds none.
__device__ __forceinline__ void wait_lgkm() { __builtin_amdgcn_s_waitcnt(0xc07f); }
__device__ __forceinline__ void barrier_seen() {
    asm volatile("" ::: "memory");
    wait_lgkm();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Eight consecutive features of one token, from sums to the stored row.
template <bool BF16, int ACT>
struct Finish {
    float ws[8], bv[8];
    __device__ __forceinline__ void features(const I8Args& a, int n) {  // n: a multiple of 8 below N
        *reinterpret_cast<floatx4*>(ws) = *reinterpret_cast<const floatx4*>(a.w_scale + n);
        *reinterpret_cast<floatx4*>(ws + 4) = *reinterpret_cast<const floatx4*>(a.w_scale + n + 4);
        if (!a.bias) {
#pragma unroll
            for (int e = 0; e < 8; ++e) bv[e] = 0.f;
        } else {
            load(a.bias, n, bv);
        }
    }
    static __device__ __forceinline__ void load(const void* p, int64_t off, float* v) {
        if constexpr (BF16) {
            const u32x4 c = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + off);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[2 * e] = lo_bf16(c[e]);
                v[2 * e + 1] = hi_bf16(c[e]);
            }
        } else {
            *reinterpret_cast<floatx4*>(v) = *reinterpret_cast<const floatx4*>(static_cast<const float*>(p) + off);
            *reinterpret_cast<floatx4*>(v + 4) = *reinterpret_cast<const floatx4*>(static_cast<const float*>(p) + off + 4);
        }
    }
    __device__ __forceinline__ void row(const I8Args& a, const int* sum, float xs, const float* res, int m, int n) const {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float z = fmaf((float)sum[e] * xs, ws[e], bv[e]);
            v[e] = BF16 ? activate_bf16<ACT>(z) : activate<ACT>(z);
            if (res) v[e] += res[e];
        }
        if constexpr (BF16) {
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.y) + (int64_t)m * a.ldy + n) =
                u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        } else {
            float* const dst = static_cast<float*>(a.y) + (int64_t)m * a.ldy + n;
            *reinterpret_cast<floatx4*>(dst) = floatx4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<floatx4*>(dst + 4) = floatx4{v[4], v[5], v[6], v[7]};
        }
    }
};

template <class C, bool BF16, int ACT>
__device__ __forceinline__ void i8_tile(const I8Args& a, int m0, int n0, int8_t* sm) {
    constexpr int TM = C::TM, TN = C::TN, FM = C::FM, FN = C::FN, ST = C::ST, G = C::G, NC = C::kCopies;
    const int wave = uni(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int l16 = lane % 16, q4 = lane / 16;
    const int wk = wave % C::WK, wm = wave / C::WK / C::WN, wn = wave / C::WK % C::WN;
    const int K = a.K, nk = (K + 127) / 128;
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x + (int64_t)m0 * a.ldx, (uint32_t)min(a.T - m0, TM) * a.ldx);
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.w + (int64_t)n0 * K, (uint32_t)min(a.N - n0, TN) * K);
    // copy c of this wave fills block id = wave * NC + c of a stage (8 rows of 128 bytes, x
    // rows first; lane l slot l: row l / 8, physical chunk l % 8, logical chunk XORed with swz2(row))
    int voff[NC], kb[NC];  // the lane's byte offset; its chunk's first k
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int b = wave * NC + c, row = (b < TM / 8 ? b : b - TM / 8) * 8 + lane / 8;
        kb[c] = ((lane % 8) ^ swz2(row)) * 16;
        voff[c] = row * (b < TM / 8 ? a.ldx : K) + kb[c];
    }
    auto issue_one = [&](int step, int8_t* st, int c) {
        const int b = wave * NC + c, k0 = step * 128;
        const int off = k0 + kb[c] < K ? voff[c] : kPast;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(b < TM / 8 ? rx : rw, (lds_void_t*)(st + b * 1024), 16, off, k0, 0, 0);
    };
    intx4 acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = intx4{0, 0, 0, 0};
    intx4 fa[2][FN], fb[2][FM];
    auto read = [&](int slot, const int8_t* st, int g) {  // the wave's g-th 64-k group of a landed stage
        const int8_t* const wb = st + TM * 128;
        const int ch = (g * C::WK + wk) * 4 + q4;
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            const int r = wn * (TN / C::WN) + i * 16 + l16;
            fa[slot][i] = *reinterpret_cast<const intx4*>(wb + r * 128 + ((ch ^ swz2(r)) * 16));
        }
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int r = wm * (TM / C::WM) + j * 16 + l16;
            fb[slot][j] = *reinterpret_cast<const intx4*>(st + r * 128 + ((ch ^ swz2(r)) * 16));
        }
    };
#pragma unroll
    for (int s = 0; s < ST; ++s)
#pragma unroll
        for (int c = 0; c < NC; ++c) issue_one(s, sm + s * C::kStage, c);
    wait_vm<(ST - 1) * NC>();
    barrier_seen();
    int8_t* st = sm;
    read(0, st, 0);
    wait_lgkm();
    // Step k's operands sit in stage k % ST; before its last group the next step's copies
    // are waited for and its first group read, and the copies of step k + ST go out
    // between the MFMAs into the stage every wave has now read.  (Group g of step k sits in
    // slot (k * G + g) % 2: with one group per step the slots alternate by step.)
    auto step = [&](int k, auto last, auto par) {
        constexpr bool kLast = decltype(last)::value;
        constexpr int kPar = decltype(par)::value;
        int8_t* const next = st + C::kStage == sm + ST * C::kStage ? sm : st + C::kStage;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int slot = (kPar * G + g) % 2;
            if (g + 1 < G) {
                read(1 - slot, st, g + 1);
            } else if constexpr (!kLast) {
                __builtin_amdgcn_sched_barrier(0);  // the MFMAs before go out ahead of the wait
                wait_vm<(ST - 2) * NC>();
                barrier_seen();
                read(1 - slot, next, 0);
            }
            __builtin_amdgcn_sched_barrier(0);  // else the reads sink below the MFMAs meant to hide them
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[slot][i], fb[slot][j], acc[i][j], 0, 0, 0);
                    if constexpr (!kLast) {
#pragma unroll
                        for (int c = 0; c < NC; ++c)
                            if (g + 1 == G && c * FM * FN / NC == i * FM + j) issue_one(k + ST, st, c);
                    }
                }
            __builtin_amdgcn_s_setprio(0);
        }
        st = next;
    };
    int k = 0;
    for (; k + 2 < nk; k += 2) {
        step(k, std::false_type{}, std::integral_constant<int, 0>{});
        step(k + 1, std::false_type{}, std::integral_constant<int, 1>{});
    }
    if (k + 1 < nk) {
        step(k, std::false_type{}, std::integral_constant<int, 0>{});
        step(k + 1, std::true_type{}, std::integral_constant<int, 1>{});
    } else {
        step(k, std::true_type{}, std::integral_constant<int, 0>{});
    }
    wait_vm<0>();  // the copies past the reduction have landed: LDS is free

    // Epilogue in slices of kRows tokens: the int32 sums go through LDS (row r's 16-byte
    // chunk c at c ^ (r & 15), one tile per k share), then each thread finishes eight features of a row at
    // a time.  Slice s holds the s-th part of every wave row's tokens.
    constexpr int kRows = C::kRows, kSlices = TM / kRows, kPart = kRows / C::WM;  // a wave row's tokens per slice
    static_assert(kPart % 16 == 0, "slices of whole blocks");
    constexpr int kCh = TN / 8, kRowStep = C::kThreads / kCh, kIt = kRows / kRowStep;
    static_assert(C::kThreads % kCh == 0 && kRows % kRowStep == 0, "row phase");
    constexpr int kSwz = TN / 4 < 16 ? TN / 4 - 1 : 15;
    const int ch = threadIdx.x % kCh, r0 = threadIdx.x / kCh, n = n0 + ch * 8, nc = min(n, a.N - 8);
    Finish<BF16, ACT> fin;
    fin.features(a, nc);
    int* const ep = reinterpret_cast<int*>(sm);
    auto slot_of = [&](int row, int c) { return row * TN + ((c ^ (row & kSwz)) * 4); };
#pragma unroll
    for (int s = 0; s < kSlices; ++s) {
        barrier_seen();
#pragma unroll
        for (int jj = 0; jj < kPart / 16; ++jj)
#pragma unroll
            for (int i = 0; i < FN; ++i)
                // acc[i][j][e]: token j*16 + l16, feature i*16 + 4 q4 + e of the wave's sub-tile
                *reinterpret_cast<intx4*>(ep + wk * kRows * TN +
                                          slot_of(wm * kPart + jj * 16 + l16, (wn * (TN / C::WN) + i * 16 + 4 * q4) >> 2)) =
                    acc[i][s * (kPart / 16) + jj];
        barrier_seen();
#pragma unroll
        for (int t = 0; t < kIt; ++t) {
            const int row = r0 + t * kRowStep, m = m0 + (row / kPart) * (TM / C::WM) + s * kPart + row % kPart;
            if (m >= a.T || n >= a.N) continue;
            int v[8];
            *reinterpret_cast<intx4*>(v) = *reinterpret_cast<const intx4*>(ep + slot_of(row, 2 * ch));
            *reinterpret_cast<intx4*>(v + 4) = *reinterpret_cast<const intx4*>(ep + slot_of(row, 2 * ch + 1));
            if constexpr (C::WK == 2) {
#pragma unroll
                for (int hc = 0; hc < 2; ++hc) {
                    const intx4 o = *reinterpret_cast<const intx4*>(ep + kRows * TN + slot_of(row, 2 * ch + hc));
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[4 * hc + e] += o[e];
                }
            }
            float res[8];
            if (a.residual) Finish<BF16, ACT>::load(a.residual, (int64_t)m * a.ldr + n, res);
            fin.row(a, v, a.x_scale[m], a.residual ? res : nullptr, m, n);
        }
    }
}

template <class C, bool BF16, int ACT>
__global__ __launch_bounds__(C::kThreads) void k_linear_i8(I8Args a, int tiles_m, int tiles_n) {
    extern __shared__ __attribute__((aligned(16))) int8_t smem_i8[];
    int tm, tn;
    tile_coords(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, tm, tn);
    i8_tile<C, BF16, ACT>(a, tm * C::TM, tn * C::TN, smem_i8);
}

template <class C, bool BF16, int ACT>
hipError_t launch_tiles(const I8Args& a, hipStream_t s) {
    auto* f = &k_linear_i8<C, BF16, ACT>;
    static bool attr_set = false;  // benign race: every thread sets the same value
    if (C::kLds > 64 * 1024 && !attr_set) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize, C::kLds);
        if (e != hipSuccess) return e;
        attr_set = true;
    }
    const int64_t tiles_m = ((int64_t)a.T + C::TM - 1) / C::TM, tiles_n = ((int64_t)a.N + C::TN - 1) / C::TN;
    if (tiles_m * tiles_n > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(f, dim3((unsigned)(tiles_m * tiles_n)), dim3(C::kThreads), C::kLds, s, a, (int)tiles_m, (int)tiles_n);
    return hipGetLastError();
}

using I8Small = I8Cfg<64, 64, 2, 2, 1, 3>;

template <bool BF16, int ACT>
hipError_t launch_form(const I8Args& a, hipStream_t s) {
    return launch_tiles<I8Small, BF16, ACT>(a, s);
}

template <bool BF16>
hipError_t launch_type(const I8Args& a, int act, hipStream_t s) {
    switch (act) {
        case 1: return launch_form<BF16, 1>(a, s);
        case 2: return launch_form<BF16, 2>(a, s);
        default: return launch_form<BF16, 0>(a, s);
    }
}

}  // namespace

hipError_t launch_linear_i8(int dtype, const int8_t* x, int ldx, const float* x_scale, const int8_t* w,
                            const float* w_scale, const void* bias, const void* residual, int ldr, int act, void* y,
                            int ldy, int T, int K, int N, hipStream_t s) {
    if (T == 0) return hipSuccess;
    const I8Args a{x, x_scale, w, w_scale, bias, residual, y, ldx, ldr, ldy, T, K, N};
    return dtype == 1 ? launch_type<true>(a, act, s) : launch_type<false>(a, act, s);
}

}  // namespace rag
