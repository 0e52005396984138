// Packed-token linear operator on 8-bit rows:
//   y = act(x_scale w_scale (x w^T) + bias) + residual
// with x int8 [T, K], w int8 [N, K], the products summed exactly in int32 on the matrix
// cores (v_mfma_i32_16x16x64_i8; K <= 131056 keeps the sums below 2^31) and scales, bias, activation and
// residual applied in fp32 to the finished sum, which is rounded to the type once.
//
// linear_kernel_i8 picks the kernel: one of its own for few tokens (further down), or TM x TN tiles, one
// per workgroup of WM x WN (x WK, over k) waves.  What bounds them:
// moving operands from L2 into LDS on the small ones (a 64 x 64 tile takes 16 KB per 0.22 us of a CU),
// the matrix cores and power on 256 x 256 ones: 8192^3 413 us, 2660 TOPS.  Operands go global -> LDS
// by bounds-checked direct copies, 128 k (one 128-byte line) of each row per stage, ST stages; the
// 16-byte chunks of a row are XOR-swizzled by it, so fragment reads of 16 rows meet distinct
// bank groups.  Rows past T or N lie outside the descriptors, chunks past K are sent past
// them: both arrive as zeros.
// A lane's fragment is 16 consecutive k of one row in both operands, and the tile is
// computed as w x^T, so that a lane ends with four consecutive features of one token.
#include <algorithm>
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
    // waves per SIMD: what the LDS lets reside
    static constexpr int kResident = 160 * 1024 / kLds < 1 ? 1 : 160 * 1024 / kLds;
    static constexpr int kWavesPerSimd = kResident * kWaves / 4 < 1 ? 1 : kResident * kWaves / 4 > 8 ? 8 : kResident * kWaves / 4;
    static_assert((TM / 8) % 2 == 0 && (TM + TN) / 8 % kWaves == 0 && kLds <= 160 * 1024 && (WK == 1 || WK == 2), "configuration");
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

// GELU's tanh form for bf16 outputs: x (1 + tanh u) / 2 = x / (1 + exp(-2u)), the hardware's power of two and
// reciprocal within two steps of fp32 (tanhf is six times the instructions: 35475 x 1024 x 4096
// 304 us with it, 214 without).
__device__ __forceinline__ float gelu_tanh_fast(float x) {
    constexpr float k = 2.0f * 0.79788456080286536f * 1.4426950408889634f;  // 2 sqrt(2 / pi) log2(e)
    const float u = x * fmaf(x * x, k * 0.044715f, k);
    return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-u));
}

template <bool BF16, int ACT>
__device__ __forceinline__ float finish_act(float x) {
    if constexpr (BF16 && ACT == 2) return gelu_tanh_fast(x);
    else if constexpr (BF16) return activate_bf16<ACT>(x);
    else return activate<ACT>(x);
}

// Eight consecutive features of one token, from sums to the stored row.
template <bool BF16, int ACT>
struct Finish {
    struct Raw {
        u32x4 v[BF16 ? 1 : 2];
    };
    static __device__ __forceinline__ Raw load(const void* p, int64_t off) {
        Raw r;
        const u32x4* const src = BF16 ? reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + off)
                                      : reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + off);
        r.v[0] = src[0];
        if constexpr (!BF16) r.v[1] = src[1];
        return r;
    }
    static __device__ __forceinline__ float get(const Raw& r, int e) {
        if constexpr (BF16) return e & 1 ? hi_bf16(r.v[0][e >> 1]) : lo_bf16(r.v[0][e >> 1]);
        else return __uint_as_float(r.v[e >> 2][e & 3]);
    }
    floatx4 ws[2];
    Raw braw;
    float bv[8];
    // the features' scales and bias: loaded here, unpacked by features() once they are used
    __device__ __forceinline__ void fetch(const I8Args& a, int n) {  // n: a multiple of 8 below N
        ws[0] = *reinterpret_cast<const floatx4*>(a.w_scale + n);
        ws[1] = *reinterpret_cast<const floatx4*>(a.w_scale + n + 4);
        if (a.bias) braw = load(a.bias, n);
    }
    __device__ __forceinline__ void features(bool bias) {
#pragma unroll
        for (int e = 0; e < 8; ++e) bv[e] = bias ? get(braw, e) : 0.f;
    }
    __device__ __forceinline__ void row(const I8Args& a, const int* sum, float xs, bool residual, const Raw& res, int m, int n) const {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf((float)sum[e] * xs, ws[e >> 2][e & 3], bv[e]);
        // The sums, up to 2^31, may pass fp32's range before the features' scales bring them back.  (One branch for
        // the wave: two ways for each lane cost 35475 x 1024 x 1024 59.0 -> 61.8 us, this nothing.)
        const bool far = fabsf(xs) > 0x1p96f;
        if (__builtin_expect(__ballot(far) != 0, 0)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = (float)fma((double)sum[e] * xs, (double)ws[e >> 2][e & 3], (double)bv[e]);
                v[e] = far ? z : v[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = finish_act<BF16, ACT>(v[e]);
        if (residual) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += get(res, e);
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
    int voff[NC], kb[2];  // the lane's byte offset; its chunk's first k, which only block parity changes
#pragma unroll
    for (int c = 0; c < 2; ++c) kb[c] = ((lane % 8) ^ swz2((wave * NC + c) * 8 + lane / 8)) * 16;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int b = wave * NC + c, row = (b < TM / 8 ? b : b - TM / 8) * 8 + lane / 8;
        voff[c] = row * (b < TM / 8 ? a.ldx : K) + kb[c & 1];
    }
    auto issue_one = [&](int step, int8_t* st, int c) {
        const int b = wave * NC + c, k0 = step * 128;
        const int off = k0 + kb[c & 1] < K ? voff[c] : kPast;
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
    // `kind` 2: such a step; 1: one of the last ST, with no copies left; 0: the last.
    auto step = [&](int k, auto kind, auto par) {
        constexpr int kKind = decltype(kind)::value;
        constexpr int kPar = decltype(par)::value;
        int8_t* const next = st + C::kStage == sm + ST * C::kStage ? sm : st + C::kStage;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int slot = (kPar * G + g) % 2;
            if (g + 1 < G) {
                read(1 - slot, st, g + 1);
            } else if constexpr (kKind > 0) {
                __builtin_amdgcn_sched_barrier(0);  // the MFMAs before go out ahead of the wait
                wait_vm<kKind == 2 ? (ST - 2) * NC : 0>();
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
                    if constexpr (kKind == 2) {
#pragma unroll
                        for (int c = 0; c < NC; ++c)
                            if (g + 1 == G && c * FM * FN / NC == i * FM + j) issue_one(k + ST, st, c);
                    }
                }
            __builtin_amdgcn_s_setprio(0);
        }
        st = next;
    };
    // The epilogue's rows: thread t finishes eight features of row t / kCh + it * kRowStep of each slice.
    constexpr int kRows = C::kRows, kSlices = TM / kRows, kPart = kRows / C::WM;  // a wave row's tokens per slice
    static_assert(kPart % 16 == 0, "slices of whole blocks");
    constexpr int kCh = TN / 8, kRowStep = C::kThreads / kCh, kIt = kRows / kRowStep;
    static_assert(C::kThreads % kCh == 0 && kRows % kRowStep == 0, "row phase");
    constexpr int kSwz = TN / 4 < 16 ? TN / 4 - 1 : 15;
    using Fin = Finish<BF16, ACT>;
    const int ch = threadIdx.x % kCh, r0 = threadIdx.x / kCh, n = n0 + ch * 8, nc = min(n, a.N - 8);
    const auto token = [&](int s, int it) {
        const int row = r0 + it * kRowStep;
        return m0 + (row / kPart) * (TM / C::WM) + s * kPart + row % kPart;
    };
    constexpr std::integral_constant<int, 0> even{}, last{};
    constexpr std::integral_constant<int, 1> odd{}, rest{};
    constexpr std::integral_constant<int, 2> copying{};
    int k = 0;
    if constexpr (G % 2 == 0) {
        // (35475 x 1024 x 1024 with residual on 64 x 64 tiles 69 us, 73 with copies past the reduction)
        for (; k + ST < nk; ++k) step(k, copying, even);
        for (; k + 1 < nk; ++k) step(k, rest, even);
        step(k, last, even);
    } else {
        // (copies past the reduction, which store zeros: a test for them in the loop cost more at K = 4096, 8.4 us and 9.2)
        for (; k + 2 < nk; k += 2) {
            step(k, copying, even);
            step(k + 1, copying, odd);
        }
        if (k + 1 < nk) {
            step(k, copying, even);
            step(k + 1, last, odd);
        } else {
            step(k, last, even);
        }
    }
    wait_vm<0>();  // the copies past the reduction have landed: LDS is free

    // Epilogue in slices of kRows tokens (slice s holds the s-th part of every wave row's):
    // the int32 sums go through LDS (row r's 16-byte chunk c at c ^ (r & 15), one tile per k
    // share), then whole rows are finished.  What it reads is loaded before the staging, at
    // indexes clamped into range: loaded under the range tests, each row's values were waited
    // for in turn.
    Fin fin;
    fin.fetch(a, nc);
    int* const ep = reinterpret_cast<int*>(sm);
    auto slot_of = [&](int row, int c) { return row * TN + ((c ^ (row & kSwz)) * 4); };
#pragma unroll
    for (int s = 0; s < kSlices; ++s) {
        float xs[kIt];
        typename Fin::Raw res[kIt];
#pragma unroll
        for (int t = 0; t < kIt; ++t) {
            const int m = min(token(s, t), a.T - 1);
            xs[t] = a.x_scale[m];
            if (a.residual) res[t] = Fin::load(a.residual, (int64_t)m * a.ldr + nc);
        }
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
        if (s == 0) fin.features(a.bias != nullptr);
#pragma unroll
        for (int t = 0; t < kIt; ++t) {
            const int row = r0 + t * kRowStep, m = token(s, t);
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
            fin.row(a, v, xs[t], a.residual != nullptr, res[t], m, n);
        }
    }
}

// Tiles of a launch in x, the rest in y: with 512 threads each 2^31 of the 2^32 - 1 that a dimension can have.
constexpr int kGridTiles = 1 << 22;

template <class C, bool BF16, int ACT>
__global__ __launch_bounds__(C::kThreads, C::kWavesPerSimd) void k_linear_i8(I8Args a, int tiles_m, int tiles_n) {
    extern __shared__ __attribute__((aligned(16))) int8_t smem_i8[];
    const int bid = blockIdx.y * kGridTiles + blockIdx.x;
    if (bid >= tiles_m * tiles_n) return;
    int tm, tn;
    tile_coords(bid, tiles_m * tiles_n, tiles_m, tiles_n, tm, tn);
    i8_tile<C, BF16, ACT>(a, tm * C::TM, tn * C::TN, smem_i8);
}

// Whole 256 x 256 tiles of a launch: all of them if the last round is nearly full, else the
// full rounds.
int64_t i8_whole_tiles(int64_t tiles, int64_t cus) {
    const int64_t rest = tiles % cus;
    return 4 * rest > 3 * cus ? tiles : tiles - rest;
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
    const int64_t tiles = tiles_m * tiles_n;
    const dim3 grid((unsigned)std::min<int64_t>(tiles, kGridTiles), (unsigned)((tiles + kGridTiles - 1) / kGridTiles));
    hipLaunchKernelGGL(f, grid, dim3(C::kThreads), C::kLds, s, a, (int)tiles_m, (int)tiles_n);
    return hipGetLastError();
}

// 256 x 256 tiles, one workgroup per CU, whole rounds of them; the tiles of the last,
// partial round run as four 128 x 128 quarters each (n_full workgroups, then the quarters).
using I8Big = I8Cfg<256, 256, 2, 4, 1, 2>;
using I8Tail = I8Cfg<128, 128, 2, 4, 1, 4>;
static_assert(I8Tail::kThreads == I8Big::kThreads && I8Tail::kLds <= I8Big::kLds, "quarters");

template <bool BF16, int ACT>
__global__ __launch_bounds__(I8Big::kThreads, 2) void k_linear_i8_big(I8Args a, int tiles_m, int tiles_n, int n_full) {
    extern __shared__ __attribute__((aligned(16))) int8_t smem_i8[];
    int tm, tn;
    if ((int)blockIdx.x < n_full) {
        tile_coords(blockIdx.x, n_full, tiles_m, tiles_n, tm, tn);
        i8_tile<I8Big, BF16, ACT>(a, tm * 256, tn * 256, smem_i8);
    } else {
        const int u = blockIdx.x - n_full;
        group_walk(n_full + u / 4, tiles_m, tiles_n, tm, tn);
        const int m0 = tm * 256 + (u & 1) * 128, n0 = tn * 256 + ((u >> 1) & 1) * 128;
        if (m0 >= a.T || n0 >= a.N) return;  // a quarter past the last token or feature
        i8_tile<I8Tail, BF16, ACT>(a, m0, n0, smem_i8);
    }
}

template <bool BF16, int ACT>
hipError_t launch_big(const I8Args& a, int cus, hipStream_t s) {
    auto* f = &k_linear_i8_big<BF16, ACT>;
    static bool attr_set = false;  // benign race: every thread sets the same value
    if (!attr_set) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize, I8Big::kLds);
        if (e != hipSuccess) return e;
        attr_set = true;
    }
    const int64_t tiles_m = ((int64_t)a.T + 255) / 256, tiles_n = ((int64_t)a.N + 255) / 256, tiles = tiles_m * tiles_n;
    const int64_t n_full = i8_whole_tiles(tiles, cus);
    if (n_full + 4 * (tiles - n_full) > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(f, dim3((unsigned)(n_full + 4 * (tiles - n_full))), dim3(I8Big::kThreads), I8Big::kLds, s, a,
                       (int)tiles_m, (int)tiles_n, (int)n_full);
    return hipGetLastError();
}

// Few tokens: 16 features per workgroup for all of at most 16 tokens, the reduction
// split over the workgroup's waves.  Bound by the weights' bytes (and latency): each is read
// once, straight into the MFMA operand, four 64-k groups per wave in flight; x comes out of L2.
constexpr int kFewGroups = 4;      // 64-k groups per wave and step
constexpr int kFewWaves = 8;       // (1 x 4096 x 1024: 4.7 us; 5.3 with four, 5.0 with sixteen)

template <bool BF16, int ACT>
__global__ __launch_bounds__(kFewWaves * kWave) void k_linear_i8_few(I8Args a) {
    __shared__ __attribute__((aligned(16))) int part[kFewWaves * 16 * 16];
    const int wave = uni(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int l16 = lane % 16, q4 = lane / 16;
    const int n0 = blockIdx.x * 16, K = a.K, steps = (K + 64 * kFewGroups - 1) / (64 * kFewGroups);
    const int8_t* const wr = a.w + (int64_t)min(n0 + l16, a.N - 1) * K;
    const int8_t* const xr = a.x + (int64_t)min(l16, a.T - 1) * a.ldx;
    intx4 acc = {0, 0, 0, 0};
    for (int s = wave; s < steps; s += kFewWaves) {
        intx4 fw[kFewGroups], fx[kFewGroups];
#pragma unroll
        for (int u = 0; u < kFewGroups; ++u) {
            const int k = (s * kFewGroups + u) * 64 + q4 * 16, kc = min(k, K - 16);
            fw[u] = *reinterpret_cast<const intx4*>(wr + kc);
            fx[u] = *reinterpret_cast<const intx4*>(xr + kc);
            if (k >= K) fw[u] = intx4{0, 0, 0, 0};  // past the reduction
        }
#pragma unroll
        for (int u = 0; u < kFewGroups; ++u) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fx[u], acc, 0, 0, 0);
    }
    // acc[e]: token l16, feature 4 q4 + e
    *reinterpret_cast<intx4*>(part + (wave * 16 + l16) * 16 + 4 * q4) = acc;
    __syncthreads();
    const int m = threadIdx.x / 2, n = n0 + 8 * (threadIdx.x % 2);
    if (m >= a.T || n >= a.N) return;
    Finish<BF16, ACT> fin;
    fin.fetch(a, n);
    const float xs = a.x_scale[m];
    typename Finish<BF16, ACT>::Raw res;
    if (a.residual) res = Finish<BF16, ACT>::load(a.residual, (int64_t)m * a.ldr + n);
    int v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
        for (int hc = 0; hc < 2; ++hc) {
            const intx4 o = *reinterpret_cast<const intx4*>(part + (w * 16 + m) * 16 + 8 * (threadIdx.x % 2) + 4 * hc);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * hc + e] += o[e];
        }
    fin.features(a.bias != nullptr);
    fin.row(a, v, xs, a.residual != nullptr, res, m, n);
}

template <bool BF16, int ACT>
hipError_t launch_few(const I8Args& a, hipStream_t s) {
    hipLaunchKernelGGL((k_linear_i8_few<BF16, ACT>), dim3((a.N + 15) / 16), dim3(kFewWaves * kWave), 0, s, a);
    return hipGetLastError();
}

template <bool BF16, int ACT>
hipError_t launch_kernel(const I8Args& a, hipStream_t s) {
    const int cus = device_cu_count();
    switch (linear_kernel_i8(a.T, a.K, a.N, ACT, BF16, cus)) {
        case kI8Few: return launch_few<BF16, ACT>(a, s);
        case kI8Tiles32x32: return launch_tiles<I8Cfg<32, 32, 1, 1, 2, 6>, BF16, ACT>(a, s);
        case kI8Tiles32x64Deep: return launch_tiles<I8Cfg<32, 64, 1, 2, 2, 6>, BF16, ACT>(a, s);
        case kI8Tiles32x64: return launch_tiles<I8Cfg<32, 64, 1, 2, 2, 4>, BF16, ACT>(a, s);
        case kI8Tiles64x64: return launch_tiles<I8Cfg<64, 64, 2, 2, 1, 3>, BF16, ACT>(a, s);
        case kI8Tiles64x128: return launch_tiles<I8Cfg<64, 128, 2, 2, 1, 3>, BF16, ACT>(a, s);
        case kI8Tiles128x128: return launch_tiles<I8Cfg<128, 128, 2, 4, 1, 2>, BF16, ACT>(a, s);
        default: return launch_big<BF16, ACT>(a, cus, s);
    }
}

template <bool BF16>
hipError_t launch_type(const I8Args& a, int act, hipStream_t s) {
    switch (act) {
        case 1: return launch_kernel<BF16, 1>(a, s);
        case 2: return launch_kernel<BF16, 2>(a, s);
        default: return launch_kernel<BF16, 0>(a, s);
    }
}

}  // namespace

// The form of tiles for a call: 0 few tokens (at most 16), 1 .. 4 tiles of 32 tokens (two k shares), 64 x 64, 64 x 128
// and 128 x 128, 5 the 256 x 256 tiles and quarters: the smallest of the modelled times in us
//     start + max(epilogue + nk * alone, rounds * (epilogue + nk * step))
// nk the 128-k steps, rounds the tiles of the busiest CU, `alone` a step's latency and `step` its
// share of a busy CU's time, the epilogue longer with an activation or fp32 outputs.  Fitted to
// 355 shapes (T 17 to 40000, K 256 to 8192, N 64 to 8192, both types, every epilogue) with 32 x 64 tiles of
// four stages as form 1.  On 240 others the kernel that linear_kernel_i8 makes of it takes 1.5% more than the
// fastest of the seven on average and 25% at worst (up to 400 tokens 1.0%).  Us on forms 1 to 5: 2237 x 2048 x 512 fp32
// 9.6, 8.9, 9.1, 14.7, 12.2; 35475 x 1024 x 4096 GELU 395, 291, 264, 225, 229; 35475 x 4096 x 1024 with residual
// 336, 225, 190, 168, 140.
int linear_form_i8(int64_t T, int64_t K, int64_t N, int act, bool bf16, int64_t cus) {
    if (T <= 16) return 0;
    struct Cost {
        int tm, tn;
        double start, epilogue, step, alone, act, f32, act32;  // act: of bf16 outputs, act32 of fp32's
    };
    static const Cost kForms[4] = {{32, 64, 2.32, 0.42, 0.158, 0.164, 0.05, 0.23, 0.31}, {64, 64, 2.38, 0.38, 0.237, 0.253, 0.14, 0.33, 0.76},
                                   {64, 128, 2.35, 0.99, 0.361, 0.361, 0.34, 0.60, 2.15}, {128, 128, 0.63, 1.98, 0.530, 0.705, 0.83, 1.05, 4.4}};
    const auto up = [](int64_t n, int64_t d) { return (n + d - 1) / d; };
    const double nk = (double)up(K, 128);
    const auto extra = [&](double a, double f, double a32) { return (bf16 ? 0.0 : f) + (!act ? 0.0 : bf16 ? a : a32); };
    // 256 x 256: rounds of whole tiles, then one of quarters
    const int64_t big = up(T, 256) * up(N, 256), whole = i8_whole_tiles(big, cus);
    const double x = extra(4.96, 4.99, 14.4);
    double best = up(whole, cus) * (10.2 + x + nk * 1.57) + up(4 * (big - whole), cus) * (4.05 + x / 4 + nk * 0.485);
    int form = 5;
    for (int i = 0; i < 4; ++i) {
        const Cost& c = kForms[i];
        const double e = c.epilogue + extra(c.act, c.f32, c.act32);
        const int64_t rounds = up(up(T, c.tm) * up(N, c.tn), cus);
        const double t = c.start + std::max(e + nk * c.alone, rounds * (e + nk * c.step));
        if (t < best) best = t, form = i + 1;
    }
    return form;
}

// The kernel of a call.  Figures are us with the weights out of the caches, and in them.
int linear_kernel_i8(int64_t T, int64_t K, int64_t N, int act, bool bf16, int64_t cus) {
    const int form = linear_form_i8(T, K, N, act, bf16, cus);
    if (form > 1) return kI8Tiles64x64 + form - 2;
    // The few tokens' workgroups read all of x for 16 features each: with more than four tokens and a GPU full of tiles
    // of 32 those are faster (8192 x 8192 with 1, 8 and 16 tokens 15.0, 14.0; 16.1, 15.1; 19.2, 17.3, and on tiles with any
    // 14.9, 12.8; 16 x 4096 x 16384 20.4, 17.6 and 16.3, 12.4), with fewer tiles they are not (16 x 4096 x 4096 7.0, 6.6 and
    // 7.7, 7.6).
    if (form == 0 && !(T > 4 && N >= 32 * cus)) return kI8Few;
    // Where the tiles of 32 tokens are fewer than the CUs each CU runs one at its own copies' latency: 32 features if that
    // many tiles still fit one round, and six stages, else 64 features and four.  On 32 x 32, 32 x 64 with six and with four
    // stages: 32 x 4096 x 4096 8.1, 10.2, 11.0 (in the caches 7.7, 7.4, 7.2); 64 x 8192 x 2048 12.3, 16.0, 18.2 (12.3, 11.5,
    // 11.4); 100 x 4096 x 4096 10.1, 8.7, 10.5 (9.3, 8.0, 7.8); 160 x 1024 x 4096, more tiles than CUs, 5.5, 5.6, 5.2 (5.5, 5.7, 5.2).
    const int64_t rows = (T + 31) / 32;
    return rows * ((N + 31) / 32) <= cus ? kI8Tiles32x32 : rows * ((N + 63) / 64) <= cus ? kI8Tiles32x64Deep : kI8Tiles32x64;
}

hipError_t launch_linear_i8(int dtype, const int8_t* x, int ldx, const float* x_scale, const int8_t* w,
                            const float* w_scale, const void* bias, const void* residual, int ldr, int act, void* y,
                            int ldy, int T, int K, int N, hipStream_t s) {
    if (T == 0) return hipSuccess;
    const I8Args a{x, x_scale, w, w_scale, bias, residual, y, ldx, ldr, ldy, T, K, N};
    return dtype == 1 ? launch_type<true>(a, act, s) : launch_type<false>(a, act, s);
}

}  // namespace rag
