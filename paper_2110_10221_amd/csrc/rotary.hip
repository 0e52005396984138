// Rotary positions of packed heads: pair i of a head turns by the angle p * inv_freq[i] at
// position p,
//   (a, b) -> amplitude * (a cos - b sin, a sin + b cos),
// positions from the plan's token map.  One read and one write of every element: bound by
// HBM bandwidth.  A workgroup takes a few tokens: the cosines and sines of a token's pairs
// are computed once into LDS and serve all its heads.  The angle is reduced in fp64: p *
// inv_freq in turns has a fraction of full fp32 accuracy up to p = 2^31, where an fp32
// product would be off by whole radians.  35475 tokens x 32 heads of 64 in bf16: 47 us alone, 60 with
// inputs out of the cache (321 MB, 5.3 TB/s: a large copy's rate); 32 single tokens 3 us, the latency of
// status, token map and row one after another.
#include "device_common.h"
#include "launch.h"

namespace rag {
namespace {

struct RotaryArgs {
    const void* x;
    void* y;
    const double* inv_freq;
    const int32_t* tok_off;
    const int32_t* tok_seq;
    const int32_t* status;
    const int32_t* pos_start;  // or NULL
    int ldx, ldy, T, heads, head_dim, rot_dim, inverse, in_place;
    float amplitude;
};

constexpr int kRotaryThreads = 256;
constexpr int kRotaryTokens = 8;     // most tokens per workgroup
constexpr int kRotaryPairs = 256;    // most pairs per head

template <bool BF16>
struct Elem;
template <>
struct Elem<true> {
    using T = uint16_t;
    static constexpr int kPer = 8;  // elements of a 16-byte chunk
    static __device__ __forceinline__ float get(T v) { return bf16_to_f32(v); }
    static __device__ __forceinline__ T put(float v) { return f32_to_bf16(v); }
    static __device__ __forceinline__ void load(const T* p, float* v) {
        const u32x4 c = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = lo_bf16(c[e]);
            v[2 * e + 1] = hi_bf16(c[e]);
        }
    }
    static __device__ __forceinline__ void store(T* p, const float* v) {
        u32x4 c;
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
        *reinterpret_cast<u32x4*>(p) = c;
    }
};
template <>
struct Elem<false> {
    using T = float;
    static constexpr int kPer = 4;
    static __device__ __forceinline__ float get(T v) { return v; }
    static __device__ __forceinline__ T put(float v) { return v; }
    static __device__ __forceinline__ void load(const T* p, float* v) {
        const floatx4 c = *reinterpret_cast<const floatx4*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = c[e];
    }
    static __device__ __forceinline__ void store(T* p, const float* v) {
        *reinterpret_cast<floatx4*>(p) = floatx4{v[0], v[1], v[2], v[3]};
    }
};

// VEC: whole 16-byte chunks (aligned rows, head_dim and the half or whole turned part
// multiples of a chunk).  HALF: pair (i, i + R/2), else (2i, 2i + 1).
template <bool BF16, bool HALF, bool VEC>
__global__ __launch_bounds__(kRotaryThreads) void k_rotary(RotaryArgs a, int tokens) {
    if (a.status[0] != 0) return;
    using E = Elem<BF16>;
    using T = typename E::T;
    constexpr int V = E::kPer;
    __shared__ __attribute__((aligned(16))) float cs[kRotaryTokens * kRotaryPairs], sn[kRotaryTokens * kRotaryPairs];
    const int t0 = blockIdx.x * tokens, nt = min(tokens, a.T - t0);
    const int R = a.rot_dim, P = R / 2, D = a.head_dim;
    const T* const x = static_cast<const T*>(a.x);
    T* const y = static_cast<T*>(a.y);
    for (int u = threadIdx.x; u < nt * P; u += kRotaryThreads) {
        const int t = t0 + u / P, i = u % P;
        const int b = a.tok_seq[t];
        const int64_t pos = (int64_t)t - a.tok_off[b] + (a.pos_start ? a.pos_start[b] : 0);
        const double turns = (double)pos * a.inv_freq[i] * 0.15915494309189533577;  // 1 / (2 pi)
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        cs[u] = a.amplitude * c;
        sn[u] = a.amplitude * (a.inverse ? -s : s);
    }
    __syncthreads();
    if constexpr (VEC && HALF) {
        // unit: chunk c of a head's first half with its partner, then the head's rest
        const int hc = P / V, rest = a.in_place ? 0 : (D - R) / V, per = hc + rest, units = a.heads * per;
        for (int u = threadIdx.x; u < nt * units; u += kRotaryThreads) {
            const int tt = u / units, w = u % units, h = w / per, c = w % per;
            const T* const xr = x + (int64_t)(t0 + tt) * a.ldx + h * D;
            T* const yr = y + (int64_t)(t0 + tt) * a.ldy + h * D;
            if (c >= hc) {
                *reinterpret_cast<u32x4*>(yr + R + (c - hc) * V) = *reinterpret_cast<const u32x4*>(xr + R + (c - hc) * V);
                continue;
            }
            float p[V], q[V], o[V], r[V];
            E::load(xr + c * V, p);
            E::load(xr + P + c * V, q);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float co = cs[tt * P + c * V + e], si = sn[tt * P + c * V + e];
                o[e] = p[e] * co - q[e] * si;
                r[e] = p[e] * si + q[e] * co;
            }
            E::store(yr + c * V, o);
            E::store(yr + P + c * V, r);
        }
    } else if constexpr (VEC) {
        const int rc = R / V, per = a.in_place ? rc : D / V, units = a.heads * per;
        for (int u = threadIdx.x; u < nt * units; u += kRotaryThreads) {
            const int tt = u / units, w = u % units, h = w / per, c = w % per;
            const T* const xr = x + (int64_t)(t0 + tt) * a.ldx + h * D + c * V;
            T* const yr = y + (int64_t)(t0 + tt) * a.ldy + h * D + c * V;
            if (c >= rc) {
                *reinterpret_cast<u32x4*>(yr) = *reinterpret_cast<const u32x4*>(xr);
                continue;
            }
            float p[V], o[V];
            E::load(xr, p);
#pragma unroll
            for (int e = 0; e < V; e += 2) {
                const float co = cs[tt * P + (c * V + e) / 2], si = sn[tt * P + (c * V + e) / 2];
                o[e] = p[e] * co - p[e + 1] * si;
                o[e + 1] = p[e] * si + p[e + 1] * co;
            }
            E::store(yr, o);
        }
    } else {
        // any even rot_dim, any alignment: one pair (or one channel of the rest) per thread
        const int rest = a.in_place ? 0 : D - R, per = P + rest, units = a.heads * per;
        for (int u = threadIdx.x; u < nt * units; u += kRotaryThreads) {
            const int tt = u / units, w = u % units, h = w / per, i = w % per;
            const T* const xr = x + (int64_t)(t0 + tt) * a.ldx + h * D;
            T* const yr = y + (int64_t)(t0 + tt) * a.ldy + h * D;
            if (i >= P) {
                yr[R + i - P] = xr[R + i - P];
                continue;
            }
            const int ia = HALF ? i : 2 * i, ib = HALF ? i + P : 2 * i + 1;
            const float p = E::get(xr[ia]), q = E::get(xr[ib]), co = cs[tt * P + i], si = sn[tt * P + i];
            yr[ia] = E::put(p * co - q * si);
            yr[ib] = E::put(p * si + q * co);
        }
    }
}

template <bool BF16>
hipError_t launch_rotary_type(const RotaryArgs& a, bool half, hipStream_t s) {
    constexpr int V = Elem<BF16>::kPer;
    const auto al16 = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    const bool vec = al16(a.x) && al16(a.y) && a.ldx % V == 0 && a.ldy % V == 0 && a.head_dim % V == 0 &&
                     (half ? a.rot_dim / 2 : a.rot_dim) % V == 0;
    // Tokens per workgroup: one where the batch has few (32 tokens x 20 heads, half turned: 3.1 us, 3.6
    // with four), else as many as give its threads a few chunks each without starving the GPU of workgroups
    // (35475 tokens in bf16 with 1, 2, 4 and 8: 2 heads 23.6, 13.5, 9.1, 6.9 us; 8 heads of 128 33.5,
    // 24.5, 23.1, 23.9; 32 heads 54.4, 46.9, 49.3, 55.9; 8 heads with 20 of 64 channels turned, one pair a
    // thread, 53.9, 44.0, 39.8, 40.8).
    const int chunks = a.heads * a.head_dim / V;  // of a token (its pairs' partners included)
    const int tokens = a.T < 1024 ? 1 : !vec ? 4 : chunks <= 32 ? 8 : chunks <= 128 ? 4 : 2;
    auto* f = half ? (vec ? &k_rotary<BF16, true, true> : &k_rotary<BF16, true, false>)
                   : (vec ? &k_rotary<BF16, false, true> : &k_rotary<BF16, false, false>);
    hipLaunchKernelGGL(f, dim3((a.T + tokens - 1) / tokens), dim3(kRotaryThreads), 0, s, a, tokens);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const PlanView& p, int dtype, const void* x, int ldx, void* y, int ldy, int heads, int head_dim,
                         int rot_dim, bool half, bool inverse, const double* inv_freq, float amplitude,
                         const int32_t* pos_start, hipStream_t s) {
    if (p.total_tokens == 0) return hipSuccess;
    const RotaryArgs a{x, y, inv_freq, p.tok_off, p.tok_seq, p.status, pos_start, ldx, ldy, p.total_tokens, heads, head_dim,
                       rot_dim, int(inverse), int(x == y), amplitude};
    return dtype == 1 ? launch_rotary_type<true>(a, half, s) : launch_rotary_type<false>(a, half, s);
}

}  // namespace rag
