// Root-mean-square norm with the residual's addition, and 8-bit rows: the norm's
// output, or any matrix, as int8 with one fp32 scale per row.
//   h = x + residual;  y = gamma * h / sqrt(mean(h^2) + eps)
//   scale = max |y| / 127;  q = rint(127 y / max |y|), the exact quotient's rounding
// A row stays in registers (16-byte chunks) between its reductions, so it is read once
// and every output is written once: the operators are bound by HBM bandwidth, and by
// latency at a few rows.  All of it is fp32; h and y are rounded to the tensor type where
// they are stored and nowhere else (the 8-bit rows come from the unrounded y).
#include <algorithm>
#include <cfloat>

#include "device_common.h"
#include "launch.h"

namespace rag {
namespace {

template <bool BF16>
struct RowChunk;  // one 16-byte chunk of a row

template <>
struct RowChunk<true> {
    static constexpr int kPer = 8;
    using Raw = u32x4;
    static __device__ __forceinline__ Raw load(const void* base, int64_t off) {
        return *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + off);
    }
    static __device__ __forceinline__ void widen(const Raw& c, float* v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = lo_bf16(c[e]);
            v[2 * e + 1] = hi_bf16(c[e]);
        }
    }
    static __device__ __forceinline__ void store(void* base, int64_t off, const float* v) {
        u32x4 c;
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(base) + off) = c;
    }
};

template <>
struct RowChunk<false> {
    static constexpr int kPer = 4;
    using Raw = floatx4;
    static __device__ __forceinline__ Raw load(const void* base, int64_t off) {
        return *reinterpret_cast<const floatx4*>(static_cast<const float*>(base) + off);
    }
    static __device__ __forceinline__ void widen(const Raw& c, float* v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = c[e];
    }
    static __device__ __forceinline__ void store(void* base, int64_t off, const float* v) {
        *reinterpret_cast<floatx4*>(static_cast<float*>(base) + off) = floatx4{v[0], v[1], v[2], v[3]};
    }
};

struct NormArgs {
    const void* x;
    const void* residual;  // or NULL
    const void* gamma;     // (norm only)
    void* sum;             // or NULL
    void* y;               // or NULL
    int8_t* q;             // or NULL
    float* q_scale;
    int ldx, ldr, lds, ldy, ldq, T, d;
    float eps;
};

// A reduction over the WPR waves of a row (its own four waves' workgroup if WPR == 4).
template <int WPR, typename Op>
__device__ __forceinline__ float row_reduce(float v, float* slots, Op op) {
    v = group_reduce<kWave>(v, op);
    if constexpr (WPR > 1) {
        const int wave = threadIdx.x / kWave;
        __syncthreads();  // the slots' previous values have been read
        if (threadIdx.x % kWave == 0) slots[wave] = v;
        __syncthreads();
        v = slots[0];
#pragma unroll
        for (int w = 1; w < WPR; ++w) v = op(v, slots[w]);
    }
    return v;
}

// Rows of a launch in x where each takes a workgroup, the rest in y: 2^24 workgroups of 256 threads in x would pass
// the 2^32 - 1 threads that a dimension can have.
constexpr int kGridRows = 1 << 20;

// WPR waves per row (1: four rows per workgroup; 4: one), at most MAXC chunks per lane.
template <bool BF16, bool NORM, int WPR, int MAXC>
__global__ __launch_bounds__(256) void k_rmsnorm(NormArgs a) {
    using IO = RowChunk<BF16>;
    constexpr int E = IO::kPer, kLanes = WPR * kWave;
    __shared__ float slots[4];
    const int row = WPR == 1 ? blockIdx.x * 4 + uni(threadIdx.x / kWave) : blockIdx.y * kGridRows + blockIdx.x;
    if (row >= a.T) return;  // (a whole workgroup, or whole waves that share nothing)
    const int lane = threadIdx.x % kLanes, nch = a.d / E;
    const auto add = [](float p, float q) { return p + q; };
    const auto max2 = [](float p, float q) { return fmaxf(p, q); };

    // every load goes out before the first value is used; indexes are clamped into the
    // row and lanes past its end hold zeros
    typename IO::Raw rx[MAXC], rr[MAXC], rg[NORM ? MAXC : 1];
#pragma unroll
    for (int c = 0; c < MAXC; ++c) {
        const int ch = min(lane + kLanes * c, nch - 1);
        rx[c] = IO::load(a.x, (int64_t)row * a.ldx + ch * E);
        if (NORM && a.residual) rr[c] = IO::load(a.residual, (int64_t)row * a.ldr + ch * E);
        if constexpr (NORM) rg[c] = IO::load(a.gamma, ch * E);
    }
    float v[MAXC][E];
#pragma unroll
    for (int c = 0; c < MAXC; ++c) {
        const int ch = lane + kLanes * c;
        IO::widen(rx[c], v[c]);
        if (NORM && a.residual) {
            float r[E];
            IO::widen(rr[c], r);
#pragma unroll
            for (int e = 0; e < E; ++e) v[c][e] += r[e];
        }
        if (ch >= nch) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[c][e] = 0.f;
        } else if (NORM && a.sum) {
            IO::store(a.sum, (int64_t)row * a.lds + ch * E, v[c]);
        }
    }
    if constexpr (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < MAXC; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) ss = fmaf(v[c][e], v[c][e], ss);
        ss = row_reduce<WPR>(ss, slots, add);
        float inv = 1.0f / sqrtf(ss / a.d + a.eps), pre = 1.0f;
        if (!(ss <= FLT_MAX)) {
            // the squares overflow (values past 1e18), or the row holds an infinity or a NaN:
            // values are taken over the largest one first
            float m = 0.f;
#pragma unroll
            for (int c = 0; c < MAXC; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) m = fmaxf(m, fabsf(v[c][e]));
            m = row_reduce<WPR>(m, slots, max2);
            if (m <= FLT_MAX) {
                pre = __builtin_amdgcn_ldexpf(1.0f, -ilogbf(m));
                ss = 0.f;
#pragma unroll
                for (int c = 0; c < MAXC; ++c)
#pragma unroll
                    for (int e = 0; e < E; ++e) ss = fmaf(v[c][e] * pre, v[c][e] * pre, ss);
                ss = row_reduce<WPR>(ss, slots, add);
                inv = 1.0f / sqrtf(ss / a.d);  // (eps is nothing beside such squares)
            }
        }
#pragma unroll
        for (int c = 0; c < MAXC; ++c) {
            float g[E];
            IO::widen(rg[c], g);
            const bool in = lane + kLanes * c < nch;
#pragma unroll
            for (int e = 0; e < E; ++e) v[c][e] = in ? g[e] * (v[c][e] * pre * inv) : 0.f;
            if (a.y && in) IO::store(a.y, (int64_t)row * a.ldy + (lane + kLanes * c) * E, v[c]);
        }
    }
    if (!a.q) return;
    float top = 0.f;  // largest magnitude; infinite if any value is not finite
#pragma unroll
    for (int c = 0; c < MAXC; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float m = fabsf(v[c][e]);
            top = fmaxf(top, m <= FLT_MAX ? m : INFINITY);
        }
    top = row_reduce<WPR>(top, slots, max2);
    float scale = top / 127.0f, mul = 127.0f / top;  // 127 / top is finite for every normal scale
    if (!(scale >= FLT_MIN)) scale = mul = 0.f;
    if (!(top <= FLT_MAX)) scale = NAN;
    const bool finite = top <= FLT_MAX;
#pragma unroll
    for (int c = 0; c < MAXC; ++c) {
        const int ch = lane + kLanes * c;
        if (ch >= nch) continue;
        float n[E], edge = 0.f;  // the integers; the largest distance of a quotient from its own
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float z = v[c][e] * mul;
            n[e] = rintf(z);
            edge = fmaxf(edge, fabsf(z - n[e]));
        }
        // A quotient this near to the middle of two steps may be on its other side, or on it (bf16 rows hold
        // exact ties by the thousand): mul and the product are each off by half a step of fp32, 2^-16 at most of
        // 127.  In fp64 z errs by 2^-44 at most, while a quotient of two fp32 values that is not a tie is 2^-34 from
        // one at least: rounded to a multiple of 2^-40 (by the added 1.5 * 2^12) every tie is one and no other is.
        if (edge > 0.5f - 0x1p-15f) {
            const double r = 127.0 / (double)top;
#pragma unroll
            for (int e = 0; e < E; ++e) n[e] = (float)rint(fma((double)v[c][e], r, 6144.0) - 6144.0);
        }
        uint32_t w[E / 4];
#pragma unroll
        for (int p = 0; p < E / 4; ++p) {
            w[p] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = finite ? (int)n[4 * p + e] : 0;
                w[p] |= (uint32_t)(i & 255) << (8 * e);
            }
        }
        int8_t* const dst = a.q + (int64_t)row * a.ldq + ch * E;
        if constexpr (E == 8) *reinterpret_cast<u32x2*>(dst) = u32x2{w[0], w[1]};
        else *reinterpret_cast<uint32_t*>(dst) = w[0];
    }
    if (lane == 0) a.q_scale[row] = scale;
}

template <bool BF16, bool NORM>
hipError_t launch_rows(const NormArgs& a, hipStream_t s) {
    constexpr int E = RowChunk<BF16>::kPer;
    const int nch = a.d / E;
    const dim3 block(256), rows(std::min(a.T, kGridRows), (a.T + kGridRows - 1) / kGridRows);
    // One wave per row up to two chunks a lane, four waves from there on, at any number of rows (us, one and
    // four; bf16 with residual, sum and 8 bits): d 512, 8 and 70312 rows 2.9, 3.3 and 39.7, 82.8; d 1024,
    // 35156 rows 38.0, 50.6; d 2048, 8 and 17578 rows 4.2, 3.4 and 38.9, 39.5; d 4096 6.0, 3.8
    // and 40.8, 38.6.
    if (nch <= kWave) hipLaunchKernelGGL((k_rmsnorm<BF16, NORM, 1, 1>), dim3((a.T + 3) / 4), block, 0, s, a);
    else if (nch <= 2 * kWave) hipLaunchKernelGGL((k_rmsnorm<BF16, NORM, 1, 2>), dim3((a.T + 3) / 4), block, 0, s, a);
    else if (nch <= 4 * kWave) hipLaunchKernelGGL((k_rmsnorm<BF16, NORM, 4, 1>), rows, block, 0, s, a);
    else if (nch <= 8 * kWave) hipLaunchKernelGGL((k_rmsnorm<BF16, NORM, 4, 2>), rows, block, 0, s, a);
    else if (nch <= 16 * kWave) hipLaunchKernelGGL((k_rmsnorm<BF16, NORM, 4, 4>), rows, block, 0, s, a);
    else if (nch <= 32 * kWave) hipLaunchKernelGGL((k_rmsnorm<BF16, NORM, 4, 8>), rows, block, 0, s, a);
    else if constexpr (!BF16)  // (bf16 rows end there)
        hipLaunchKernelGGL((k_rmsnorm<BF16, NORM, 4, 16>), rows, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm(int dtype, const void* x, int ldx, const void* residual, int ldr, const void* gamma, float eps,
                          void* sum, int lds, void* y, int ldy, int8_t* q, int ldq, float* q_scale, int T, int d,
                          hipStream_t s) {
    if (T == 0) return hipSuccess;
    const NormArgs a{x, residual, gamma, sum, y, q, q_scale, ldx, ldr, lds, ldy, ldq, T, d, eps};
    return dtype == 1 ? launch_rows<true, true>(a, s) : launch_rows<false, true>(a, s);
}

hipError_t launch_quantize_i8(int dtype, const void* x, int ldx, int8_t* q, int ldq, float* scale, int T, int d,
                              hipStream_t s) {
    if (T == 0) return hipSuccess;
    const NormArgs a{x, nullptr, nullptr, nullptr, nullptr, q, scale, ldx, 0, 0, 0, ldq, T, d, 0.f};
    return dtype == 1 ? launch_rows<true, false>(a, s) : launch_rows<false, false>(a, s);
}

}  // namespace rag
