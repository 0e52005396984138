// Causal attention with a sliding window and first tokens that stay visible, over the
// packed batch or over a cache: position p sees the keys j <= p with j > p - window or
// j < sinks.
//
// One pass over the keys that some row of an item sees, like the fused ragged attention
// (attention.hip): chunks of 32 keys through two LDS stages, S^T = K Q^T in fp32, a running
// reference m and sum of the softmax, O^T += V^T E^T, one division at the end.
//   items   the entries of the plan's Attn.V list, 64 rows per workgroup of two waves (or
//           two entries, 128 rows and four waves).  A
//           row is a (token, query head) pair: the G heads that share a key head
//           are consecutive rows, so their keys are read once and a step of
//           single tokens fills rows with heads.  Entry (b, h, ti) is tile (h % G) *
//           ceil(L_b / 64) + ti of key head h / G, from its last tile to its first (those that see
//           most start first: two sequences of 8192 tokens, all visible, 500 us, 491 so);
//           entries past them return.
//   chunks  of a tile: those of the window from the last to the first, then the sinks'.
//           Downwards because a row's own key is always visible: the first chunk then
//           sets nearly every row's reference, where upwards the rows whose
//           window begins later would raise theirs from nothing, a recomputation each tile.
//   masks   only in chunks that cut some row's range; a chunk no row of a wave sees is
//           skipped by it.  Hidden values are multiplied by a zero, so those that are not
//           finite are taken out of such a chunk's operand and given to the rows that see
//           them after the last chunk (in the loop their handling cost 35 registers, the
//           fourth wave per SIMD: six prompts of 1500 to 8192 tokens 172 us, 161 without, when
//           it was moved).  The masks are bits of a word per row and chunk (166 us, 161).
//   splits  where few rows meet many keys the chunks are dealt to several workgroups
//           (blockIdx.y), whose (reference, sum, output) states a second launch joins.
// Nothing is rounded but the result.  In bf16 the P V product takes each exponential as two bf16
// values, its rounding and the rest (2^-16 of it is lost): the result is 1.65e-3 from the exact one
// by its norm, its own rounding, where one value gives 2.29e-3 (six prompts of 1500 to 8192 tokens,
// window 1024, 16/4 heads, 145 us with one, 186 with two; two of 8192, all visible, 16/8 heads, 436 and 581;
// 32 single tokens 31.1 either way, they wait for memory; the times above are with one).  fp32
// products run on v_mfma_f32_16x16x4f32, 16 keys (4 for P V) by 16 rows at a time, and only
// those that any row sees: a window of 96 is 111 keys to 16 rows, to 32 x 32 blocks it was 160 (a tenth of the time of
// batch 32 of 16 to 512 tokens, 8 heads, and of 64 single tokens, caches to 2048, 8 heads; six prompts
// of 1500 to 8192 tokens, window 1024, take 2% more).
// What bounds it: for prompts the vector instructions and the MFMAs, whose cycles add up to the launch (60% and
// 41% of a SIMD's: 552 and 384 for a chunk and wave, of 927), for they do not pass under one another (six
// prompts of 1500 to 8192 tokens, window 1024, 16/4 heads: 186 us, 550 TFLOP/s of visible pairs).  In fp32 latency: batch 32 of
// 16 to 512 tokens, window 96, 8 heads, 40 us, has its matrix units busy for 24% of the time and its vector units for 9%, with 1.1
// waves on a SIMD (179 registers allow two, and 1200 workgroups are a round of 1024 and the start of another).  For single
// tokens the bytes of K and V: 32 tokens over 4100 keys of 4 heads each, 134 MB, 28 us (4.8 TB/s; a
// large copy reaches 5.2) and 4.5 for the join.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "attention_common.h"
#include "launch.h"

namespace rag {
namespace {

constexpr int kWinBlock = 32;       // rows per wave
constexpr int kWinChunk = 32;       // keys per LDS stage

struct WinArgs {
    const int32_t* lengths;
    const int32_t* tok_off;
    const int32_t* av_items;
    int64_t av_cap;
    int32_t* status;
    const int64_t* kv_first;  // NULL: the packed batch's own rows
    const int32_t* kv_len;
    int64_t kv_rows;
    int max_kv;
    const void *q, *k, *v;
    void* out;
    int ldq, ldk, ldv, ldo;
    int heads, group;  // query heads; query heads per key head
    uint32_t magic;    // 2^32 / group, rounded up (0 for a group of one)
    int window, sinks;
    float scale;
    int T, splits;
    int stride;      // between the list entries that hold rows: G where no sequence has more than one tile a key head, 2 of 128-row tiles
    int dealt;       // entries go to the XCDs in runs (else one by one)
    float* part_o;   // [splits][T][heads][64] unnormalised outputs
    float* part_ml;  // [splits][T][heads][2] reference and sum
};

template <bool BF16>
struct WinT;
template <>
struct WinT<true> {
    using T = uint16_t;
    static constexpr int kRow = 128, kChunks = 8;  // bytes and 16-byte chunks of a row
    static __device__ __forceinline__ int swz(int row) { return kv_swz(row); }
};
template <>
struct WinT<false> {
    using T = float;
    static constexpr int kRow = 256, kChunks = 16;
    // (16 rows in any order, and rows q apart by 64 bytes: K fragments and V columns meet all banks)
    static __device__ __forceinline__ int swz(int row) { return (row & 3) << 2 | (row >> 2 & 3); }
};

// Entry of a workgroup where neighbours go to one XCD in runs of kStreamRun.
__device__ __forceinline__ int64_t dealt_item(int64_t bid) {
    const int64_t xcd = bid % 8, j = bid / 8;
    return ((j / kStreamRun) * 8 + xcd) * kStreamRun + j % kStreamRun;
}

// The last key before position p's window (keys above it are in the window), at least -1.
__device__ __forceinline__ int window_below(int p, int window) {
    return (int)max((int64_t)p - window, (int64_t)-1);
}

__device__ __forceinline__ floatx4 mfma16x16x4(float a, float b, const floatx4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t chunk_rsrc(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}

__device__ __forceinline__ void copy_1k(__amdgpu_buffer_rsrc_t r, void* dst, int off) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)dst, 16, off, 0, 0, 0);
}

__device__ __forceinline__ bool finite_f32(float v) { return fabsf(v) <= FLT_MAX; }

template <bool BF16, int NW>
__global__ __launch_bounds__(NW * kWave, BF16 ? 4 : 2)
void k_attention_window(WinArgs a) {
    using W = WinT<BF16>;
    using T = typename W::T;
    constexpr int kRows = NW * kWinBlock;                  // rows of a tile
    constexpr int kStage = 2 * kWinChunk * W::kRow;        // K rows, then V rows
    constexpr int kBlockRows = 1024 / W::kRow;             // rows of a 1 KB copy
    constexpr int kBlocks = kWinChunk / kBlockRows / NW;  // copies of K (and of V) per wave and chunk
    constexpr int kEs = (int)sizeof(T);
    __shared__ __attribute__((aligned(16))) uint8_t kvs[2 * kStage];
    const int wave = uni(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    // A lane holds scores of one row in each of RB blocks of LR rows, of the keys that its `part` says:
    // score r is key 8 (r / 4) + 4 part + r % 4 in bf16 and 16 (r / 4) + 4 (r % 4) + part in fp32.
    constexpr int RB = BF16 ? 1 : 2, LR = kWinBlock / RB, NS = 16 / RB;
    const int lrow = lane % LR, part = lane / LR;
    const float zs = softmax_factor(a.scale);
    const bool flip = a.scale < 0.f;
    const int G = a.group;
    // LDS addresses of the transposed V reads in stage 0, key step 0: within 16 lanes, lane 4 e + q
    // addresses row e, columns 4 q .. 4 q + 3 of a 4 x 16 block and receives column (lane % 16)
    uint32_t vaddr[2][2];
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi)
            vaddr[cb][hi] = (uint32_t)(uintptr_t)(lds_void_t*)kvs +
                            2 * kv_off(4 * (lane / 32) + (lane % 16) / 4 + 8 * hi, 32 * cb + 16 * (lane / 16 % 2) + 4 * (lane % 4));

    const int64_t bid = (int64_t)blockIdx.z * gridDim.x + blockIdx.x;
    const int64_t it = (a.dealt ? dealt_item(bid) : bid) * a.stride;
    // (each group's loads go out together: an item's start is a chain of three)
    const int32_t* const entry = a.av_items + 3 * min(it, a.av_cap - 1);
    const int errors = a.status[0], n_items = a.status[2], eb = entry[0], eh = entry[1], eti = entry[2];
    if (uni(errors) != 0 || it >= uni(n_items)) return;
    const int seq = uni(eb), h = uni(eh), ti = uni(eti);
    const int len = a.lengths[seq], off = a.tok_off[seq], kvn = a.kv_len ? a.kv_len[seq] : len;
    const int64_t kv0 = a.kv_len ? a.kv_first[seq] : off;
    const int L = uni(len), t0 = uni(off);
    const auto per_group = [&](int x) { return G == 1 ? x : (int)__umulhi((uint32_t)x, a.magic); };  // x / G, x < 2^16
    const int hk = uni(per_group(h)), rows = L * G;
    const int entry_no = (h - hk * G) * ((L + kTile - 1) / kTile) + ti;  // of the sequence and key head
    const int r0 = ((rows - 1) / kRows - entry_no / (kRows / kTile)) * kRows;
    if (r0 < 0) return;
    const int n = uni(kvn);  // keys
    const int64_t first = uni64(kv0);
    if (a.kv_len) {
        if (n < 0 || n > a.max_kv || first < 0 || first > a.kv_rows - n) {
            if (threadIdx.x == 0) atomicOr(a.status, kDataKvRange);
            return;
        }
    }
    const int past = n - L;  // position of token 0
    // the tile's positions
    const int tok0 = uni(G == 1 ? r0 : r0 / G), rem = r0 - tok0 * G;  // the tile's first row
    const auto token = [&](int row) { return min(tok0 + per_group(rem + row), L - 1); };  // of a row of the tile
    const int tlo = past + tok0, thi = past + uni(token(kRows - 1));
    // chunks: window [cw0, cw1) downwards, then the sinks' [0, cs) below them
    int cw0 = (window_below(tlo, a.window) + 1) / kWinChunk, cw1 = thi / kWinChunk + 1;
    if (thi < 0 || a.window == 0) cw0 = cw1 = INT32_MAX / kWinChunk;
    const int seen_sinks = min(a.sinks, thi + 1);
    const int cs = seen_sinks > 0 ? min((seen_sinks + kWinChunk - 1) / kWinChunk, cw0) : 0;
    const int nwin = cw1 - cw0, nch = nwin + cs;
    const int per = (nch + a.splits - 1) / a.splits;
    const int i0 = min(nch, (int)blockIdx.y * per), i1 = min(nch, i0 + per);
    const auto chunk = [&](int i) { return i < nwin ? cw1 - 1 - i : cs - 1 - (i - nwin); };
    const int sinks1 = a.sinks / kWinChunk + (a.sinks % kWinChunk != 0);  // chunks from here on hold no sink
    // A row at position p sees the `range` keys from `from` on and those below sink_range.  Of the wave's rows: the
    // last chunk that any sees (-1: none) and the first of the windows; chunks [whole0, whole1)
    // are seen whole by all.
    const int w0 = wave * kWinBlock;
    const bool active = r0 + w0 < rows;
    int tok[RB], head[RB], p[RB], from[RB], sink_range[RB];
    uint32_t range[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int row = min(w0 + LR * b + lrow, rows - 1 - r0);
        tok[b] = token(row);
        head[b] = hk * G + (rem + row - (tok[b] - tok0) * G);
        p[b] = past + tok[b];
        from[b] = window_below(p[b], a.window) + 1;
        range[b] = (uint32_t)max(p[b] + 1 - from[b], 0);
        sink_range[b] = min(a.sinks, p[b] + 1);
    }
    const int plo = past + uni(token(w0)), phi = past + uni(token(w0 + kWinBlock - 1));
    const int last = active && phi >= 0 ? phi / kWinChunk : -1, wfrom = window_below(plo, a.window) + 1, wfirst = wfrom / kWinChunk;
    // of a block of LR rows: does any see one of the n keys from k0 on?
    const int bhi[2] = {past + uni(token(w0 + LR - 1)), r0 + w0 + kWinBlock - LR < rows ? phi : -1};  // (-1: no rows)
    const int bfrom[2] = {wfrom, window_below(past + uni(token(w0 + kWinBlock - LR)), a.window) + 1};
    const auto block_sees = [&](int b, int k0, int n) { return k0 <= bhi[b] && (k0 + n > bfrom[b] || k0 < a.sinks); };
    const int whole0 = (window_below(phi, a.window) + kWinChunk) / kWinChunk, whole1 = plo >= 0 ? (plo + 1) / kWinChunk : 0;

    // copy i of this wave fills rows 1 KB apart from block wave * kBlocks + i of K and V;
    // rows past the last key arrive as zeros.  The descriptor starts at the chunk, so a
    // cache of any size is in reach.
    int vko[kBlocks], vvo[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
        const int r = (wave * kBlocks + i) * kBlockRows + lane / W::kChunks;
        const int c = ((lane % W::kChunks) ^ W::swz(r)) * 16;
        vko[i] = r * a.ldk * kEs + c;
        vvo[i] = r * a.ldv * kEs + c;
    }
    const T* const kbase = static_cast<const T*>(a.k) + first * a.ldk + hk * kHeadDim;
    const T* const vbase = static_cast<const T*>(a.v) + first * a.ldv + hk * kHeadDim;
    const int tail_chunk = n / kWinChunk, tail = n % kWinChunk;  // the chunk that the last key cuts
    const auto issue = [&](int i, int stage) {
        const int c = chunk(i), valid = c == tail_chunk ? tail : kWinChunk;
        const __amdgpu_buffer_rsrc_t rk = chunk_rsrc(kbase + (int64_t)c * (kWinChunk * a.ldk), (uint32_t)(valid * a.ldk) * kEs);
        const __amdgpu_buffer_rsrc_t rv = chunk_rsrc(vbase + (int64_t)c * (kWinChunk * a.ldv), (uint32_t)(valid * a.ldv) * kEs);
        uint8_t* const st = kvs + stage;
#pragma unroll
        for (int i2 = 0; i2 < kBlocks; ++i2) {
            const int blk = wave * kBlocks + i2;
            copy_1k(rk, st + blk * 1024, vko[i2]);
            copy_1k(rv, st + kWinChunk * W::kRow + blk * 1024, vvo[i2]);
        }
    };
    // Q operand: channels 16 u + 8 part .. in bf16, 16 u + 4 part + e in fp32
    u32x4 qf[RB][4];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const T* const qrow = static_cast<const T*>(a.q) + (int64_t)(t0 + tok[b]) * a.ldq + head[b] * kHeadDim;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            qf[b][u] = active ? *reinterpret_cast<const u32x4*>(qrow + 16 * u + (BF16 ? 8 : 4) * part) : u32x4{0u, 0u, 0u, 0u};
            if (flip) qf[b][u] ^= BF16 ? 0x80008000u : 0x80000000u;
        }
    }
    float m[RB], lsum[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) m[b] = -FLT_MAX, lsum[b] = 0.f;
    int fresh = 1;  // no chunk yet (a bool would be a lane mask)
    bool infinite = false;  // a chunk with hidden keys held values that are not finite
    // O^T: NO blocks of WO channels (32 of one row block, 16 of each of two); register e of block cb is channel
    // WO cb + 8 (e / 4) + 4 part + e % 4
    constexpr int NO = BF16 ? 2 : 4, WO = kHeadDim / NO, EO = BF16 ? 16 : 4;
    using Out = std::conditional_t<BF16, floatx16, floatx4>;
    Out oacc[RB][NO];
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int cb = 0; cb < NO; ++cb)
#pragma unroll
            for (int e = 0; e < EO; ++e) oacc[b][cb][e] = 0.f;

    const auto sees = [&](int b, int j) { return ((uint32_t)(j - from[b]) < range[b]) | (j < sink_range[b]); };
    // One chunk of the stage at byte `stage`; `whole`: every row sees all of it.
    const auto work = [&](int c, bool whole, auto stg) {
        constexpr int stage = decltype(stg)::value;
        const int c0 = c * kWinChunk;
        const uint8_t* const kst = kvs + stage;
        const uint8_t* const vst = kst + kWinChunk * W::kRow;
        float sc[RB][NS];
        // (`again`: the rare recomputation, where V is already held and K is read as registers allow)
        const auto products = [&](auto again) {
            if constexpr (BF16) {
                const uint16_t* const ks = reinterpret_cast<const uint16_t*>(kst);
                u32x4 kf[4];
                floatx16 acc;
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r] = 0.f;
#pragma unroll
                for (int u = 0; u < 4; ++u) kf[u] = *reinterpret_cast<const u32x4*>(ks + kv_off(lrow, 16 * u + 8 * part));
                if constexpr (!decltype(again)::value) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int u = 0; u < 4; ++u) acc = mfma32x32x16(as_bf16x8(kf[u]), as_bf16x8(qf[0][u]), acc);
#pragma unroll
                for (int r = 0; r < 16; ++r) sc[0][r] = acc[r];
            } else {
                // 16 keys by 16 rows at a time, where any row sees a key of them; operand row i is key 4 (i % 4) + i / 4
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const int kk = 16 * kb + 4 * (lrow % 4) + lrow / 4;
                    floatx4 kf[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        kf[u] = *reinterpret_cast<const floatx4*>(kst + kk * W::kRow + (((4 * u + part) ^ W::swz(kk)) * 16));
                    floatx4 acc[RB];
                    const auto multiply = [&](int b0, int b1) {
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
#pragma unroll
                                for (int b = b0; b < b1; ++b) acc[b] = mfma16x16x4(kf[u][e], __builtin_bit_cast(floatx4, qf[b][u])[e], acc[b]);
                    };
#pragma unroll
                    for (int b = 0; b < RB; ++b) acc[b] = floatx4{0.f, 0.f, 0.f, 0.f};
                    const bool first = block_sees(0, c0 + 16 * kb, 16), second = block_sees(1, c0 + 16 * kb, 16);
                    if (first && second) multiply(0, 2);  // (two chains of dependent products in turn)
                    else if (first) multiply(0, 1);
                    else if (second) multiply(1, 2);
#pragma unroll
                    for (int b = 0; b < RB; ++b)
#pragma unroll
                        for (int r = 0; r < 4; ++r) sc[b][4 * kb + r] = acc[b][r];
                }
            }
        };
        const auto hide = [&] {
            if (!whole) {
                // bit j: key c0 + j (past the part's first) is seen
                const auto below = [](int n) { return n >= 32 ? ~0u : ~(~0u << max(n, 0)); };
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    const uint32_t seen = ((below(p[b] + 1 - c0) & ~below(from[b] - c0)) | below(sink_range[b] - c0)) >> (BF16 ? 4 * part : part);
#pragma unroll
                    for (int r = 0; r < NS; ++r) {
                        const uint32_t all = (uint32_t)__builtin_amdgcn_sbfe((int)seen, BF16 ? 8 * (r / 4) + r % 4 : 16 * (r / 4) + 4 * (r % 4), 1);  // or no bits
                        sc[b][r] = __uint_as_float((all & __float_as_uint(sc[b][r])) | (~all & 0xff800000u));
                    }
                }
            }
        };
        const auto chunk_max = [&](int b) {
            float cmax = sc[b][0];
#pragma unroll
            for (int r = 1; r < NS; ++r) cmax = fmaxf(cmax, sc[b][r]);
            if constexpr (!BF16) cmax = fmaxf(cmax, __shfl_xor(cmax, 16));
            return max_xor32(cmax) * zs;
        };
        const auto exps = [&](int b) {
#pragma unroll
            for (int r = 0; r < NS; ++r) sc[b][r] = __builtin_amdgcn_exp2f(fmaf(sc[b][r], zs, -m[b]));
            float t[NS / 2];
#pragma unroll
            for (int r = 0; r < NS / 2; ++r) t[r] = sc[b][2 * r] + sc[b][2 * r + 1];
#pragma unroll
            for (int d = NS / 4; d > 0; d /= 2)
#pragma unroll
                for (int r = 0; r < d; ++r) t[r] += t[r + d];
            return t[0];
        };
        products(std::false_type{});
        // V^T operand: the lane's keys 16 t + {4 part .. + 3, 8 + 4 part .. + 3} of channel 32 cb + lrow, by transposed
        // reads whose latency passes under the products above (inline assembly, its own wait
        // included: at the builtin the compiler waits for every copy into LDS, the next chunk's
        // too)
        u32x2 tr[2][2][2];
        if constexpr (BF16) {
            __builtin_amdgcn_sched_barrier(0);
            asm volatile(
                "ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
                "ds_read_b64_tr_b16 %1, %9 offset:%12\n\t"
                "ds_read_b64_tr_b16 %2, %10 offset:%12\n\t"
                "ds_read_b64_tr_b16 %3, %11 offset:%12\n\t"
                "ds_read_b64_tr_b16 %4, %8 offset:%13\n\t"
                "ds_read_b64_tr_b16 %5, %9 offset:%13\n\t"
                "ds_read_b64_tr_b16 %6, %10 offset:%13\n\t"
                "ds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(tr[0][0][0]), "=&v"(tr[0][0][1]), "=&v"(tr[0][1][0]), "=&v"(tr[0][1][1]),
                  "=&v"(tr[1][0][0]), "=&v"(tr[1][0][1]), "=&v"(tr[1][1][0]), "=&v"(tr[1][1][1])
                : "v"(vaddr[0][0]), "v"(vaddr[0][1]), "v"(vaddr[1][0]), "v"(vaddr[1][1]),
                  "i"(stage + kWinChunk * W::kRow), "i"(stage + kWinChunk * W::kRow + 16 * W::kRow)
                : "memory");
        }
        hide();
        fresh = uni(fresh);
        if (fresh) {  // (no visible key: any later score is far above)
#pragma unroll
            for (int b = 0; b < RB; ++b) m[b] = fmaxf(chunk_max(b), -FLT_MAX);
        }
        float ps[RB];
        bool over = false;
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            ps[b] = exps(b);
            over |= !(ps[b] <= kSumCap);
        }
        // a lane sum above kSumCap (or NaN) means a score well above m: raise m to the
        // chunk's maximum and rescale what has been summed
        if (!fresh && __ballot(over) != 0) {
            products(std::true_type{});
            hide();
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const float mn = fmaxf(m[b], chunk_max(b));
                const float alpha = __builtin_amdgcn_exp2f(m[b] - mn);
                lsum[b] *= alpha;
#pragma unroll
                for (int cb = 0; cb < NO; ++cb)
#pragma unroll
                    for (int e = 0; e < EO; ++e) oacc[b][cb][e] *= alpha;
                m[b] = mn;
                ps[b] = exps(b);
            }
        }
        fresh = 0;
#pragma unroll
        for (int b = 0; b < RB; ++b) lsum[b] += ps[b];
        // Values that are not finite, among hidden keys, would reach every row (0 times infinity): they
        // are taken out of the operand here and looked for after the last chunk.
        if constexpr (BF16) {
            if (!whole) {
                typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
                u16x2 top = {0, 0};  // largest exponents: all ones if not finite
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, tr[e >> 3][e >> 2 & 1][e >> 1 & 1][e & 1] & 0x7f807f80u));
                if (__ballot(max(top[0], top[1]) == 0x7f80) != 0) {
                    infinite = true;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        uint32_t x = tr[e >> 3][e >> 2 & 1][e >> 1 & 1][e & 1];
                        if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
                        if ((x & 0x7f800000u) == 0x7f800000u) x &= 0x0000ffffu;
                        tr[e >> 3][e >> 2 & 1][e >> 1 & 1][e & 1] = x;
                    }
                }
            }
            __builtin_amdgcn_s_setprio(1);  // (matrix instructions of one wave beside the others' vector work)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                u32x4 high, low;  // an exponential as two bf16
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p0 = sc[0][8 * t + 2 * e], p1 = sc[0][8 * t + 2 * e + 1];
                    high[e] = pack_bf16x2(p0, p1);
                    low[e] = pack_bf16x2(p0 - lo_bf16(high[e]), p1 - hi_bf16(high[e]));
                }
                const auto multiply = [&](const u32x4& p) {
#pragma unroll
                    for (int cb = 0; cb < 2; ++cb)
                        oacc[0][cb] = mfma32x32x16(as_bf16x8(u32x4{tr[t][cb][0][0], tr[t][cb][0][1], tr[t][cb][1][0], tr[t][cb][1][1]}),
                                                   as_bf16x8(p), oacc[0][cb]);
                };
                multiply(high);
                multiply(low);
            }
            __builtin_amdgcn_s_setprio(0);
        } else {
            // keys 4 r + part of channel 16 cb + lrow
            float vf[NS][NO];
#pragma unroll
            for (int r = 0; r < NS; ++r)
#pragma unroll
                for (int cb = 0; cb < NO; ++cb) {
                    const int kk = 4 * r + part, ch = 16 * cb + lrow;
                    vf[r][cb] = *reinterpret_cast<const float*>(vst + kk * W::kRow + (((ch >> 2) ^ W::swz(kk)) * 16) + (ch & 3) * 4);
                }
            if (!whole) {
                uint32_t top = 0;  // largest magnitude's bits (those of values that are not finite from 0x7f800000 on)
#pragma unroll
                for (int r = 0; r < NS; ++r)
#pragma unroll
                    for (int cb = 0; cb < NO; ++cb) top = max(top, __float_as_uint(vf[r][cb]) & 0x7fffffffu);
                if (__ballot(top >= 0x7f800000u) != 0) {
                    infinite = true;
#pragma unroll
                    for (int r = 0; r < NS; ++r)
#pragma unroll
                        for (int cb = 0; cb < NO; ++cb)
                            if (!finite_f32(vf[r][cb])) vf[r][cb] = 0.f;
                }
            }
            // four keys at a time, where any row of the block sees one
#pragma unroll
            for (int r = 0; r < NS; ++r)
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    if (!block_sees(b, c0 + 4 * r, 4)) continue;
#pragma unroll
                    for (int cb = 0; cb < NO; ++cb) oacc[b][cb] = mfma16x16x4(vf[r][cb], sc[b][r], oacc[b][cb]);
                }
        }
    };
    const auto step = [&](int i, auto stg) {
        constexpr int stage = decltype(stg)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's copies of chunk i
        attn_barrier();  // ... and the other waves'; the other stage was last read in step i - 1
        if (i + 1 < i1) issue(i + 1, stage ^ kStage);
        const int c = chunk(i);
        if (c > last || (c < wfirst && c >= sinks1)) return;  // no row of the wave sees a key of it
        work(c, c >= whole0 && c < whole1, stg);
    };
    if (i0 < i1) issue(i0, 0);
    for (int i = i0; i < i1; i += 2) {
        step(i, std::integral_constant<int, 0>{});
        if (i + 1 < i1) step(i + 1, std::integral_constant<int, kStage>{});
    }
    // Values that are not finite: a positive weight leaves them what they are, where products with an
    // exponential's second part, or with one too small for fp32, may be NaN.  Outputs that are not finite are
    // looked into too (unless the row's weights are not: a NaN stays).
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        float odd[4] = {0.f, 0.f, 0.f, 0.f};  // NaN with any
#pragma unroll
        for (int cb = 0; cb < NO; ++cb)
#pragma unroll
            for (int e = 0; e < EO; ++e) odd[e % 4] = fmaf(oacc[b][cb][e], 0.f, odd[e % 4]);
        const float all = (odd[0] + odd[1]) + (odd[2] + odd[3]);
        infinite |= all != all && finite_f32(lsum[b]);
    }
    if (__builtin_expect(__ballot(infinite) != 0, 0)) {
        Out found[RB][NO];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int cb = 0; cb < NO; ++cb)
#pragma unroll
                for (int e = 0; e < EO; ++e) found[b][cb][e] = 0.f;
        for (int i = i0; i < i1; ++i) {
            for (int j = chunk(i) * kWinChunk, j1 = j + kWinChunk; j < j1; ++j) {
                const T* const vrow = vbase + (int64_t)j * a.ldv + 4 * part;
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    if (!sees(b, j)) continue;
#pragma unroll
                    for (int cb = 0; cb < NO; ++cb)
#pragma unroll
                        for (int e = 0; e < EO; ++e) {
                            float x;
                            if constexpr (BF16) x = bf16_to_f32(vrow[WO * cb + 8 * (e / 4) + e % 4]);
                            else x = vrow[WO * cb + e];
                            if (!finite_f32(x)) found[b][cb][e] += x;
                        }
                }
            }
        }
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int cb = 0; cb < NO; ++cb)
#pragma unroll
                for (int e = 0; e < EO; ++e)
                    if (found[b][cb][e] != 0.f && finite_f32(lsum[b])) oacc[b][cb][e] = found[b][cb][e];
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        if constexpr (!BF16) lsum[b] += __shfl_xor(lsum[b], 16);
        lsum[b] = sum_xor32(lsum[b]);
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        float sum = lsum[b];
        if (r0 + w0 + LR * b + lrow >= rows) continue;
        if (p[b] < 0 || (a.window == 0 && a.sinks == 0)) sum = 1.f;  // the row sees nothing: its output is zero
        const int64_t gr = (int64_t)(t0 + tok[b]);
        if (a.splits > 1) {
            const int64_t slot = ((int64_t)blockIdx.y * a.T + gr) * a.heads + head[b];
            float* const po = a.part_o + slot * kHeadDim;
#pragma unroll
            for (int cb = 0; cb < NO; ++cb)
#pragma unroll
                for (int g = 0; g < EO / 4; ++g)
                    *reinterpret_cast<floatx4*>(po + WO * cb + 8 * g + 4 * part) =
                        floatx4{oacc[b][cb][4 * g], oacc[b][cb][4 * g + 1], oacc[b][cb][4 * g + 2], oacc[b][cb][4 * g + 3]};
            if (part == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * slot) = float2{m[b], sum};
        } else {
            const float inv = 1.0f / sum;
            T* const orow = static_cast<T*>(a.out) + gr * a.ldo + head[b] * kHeadDim;
#pragma unroll
            for (int cb = 0; cb < NO; ++cb)
#pragma unroll
                for (int g = 0; g < EO / 4; ++g) {
                    const float o0 = oacc[b][cb][4 * g] * inv, o1 = oacc[b][cb][4 * g + 1] * inv, o2 = oacc[b][cb][4 * g + 2] * inv,
                                o3 = oacc[b][cb][4 * g + 3] * inv;
                    T* const dst = orow + WO * cb + 8 * g + 4 * part;
                    if constexpr (BF16) *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16x2(o0, o1), pack_bf16x2(o2, o3)};
                    else *reinterpret_cast<floatx4*>(dst) = floatx4{o0, o1, o2, o3};
                }
        }
    }
}

// Joins the splits' states of a (token, head) row: sixteen lanes of four channels each, all
// their PER loads in flight at once.  GROUPS = 16: one row per workgroup, whose sixteen groups take every
// sixteenth split; GROUPS = 1: sixteen rows.
constexpr int kWinMaxSplits = 256;

template <bool BF16, int GROUPS, int PER>
__global__ __launch_bounds__(256) void k_attention_window_join(WinArgs a) {
    if (a.status[0] != 0) return;
    using T = typename WinT<BF16>::T;
    __shared__ float wmax[4], wsum[4];
    __shared__ __attribute__((aligned(16))) float wout[4][kHeadDim];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, c = lane % 16 * 4;
    const int64_t rows = (int64_t)a.T * a.heads;
    const int64_t r = GROUPS == 1 ? (int64_t)blockIdx.x * 16 + threadIdx.x / 16 : blockIdx.x;
    const int g = GROUPS == 1 ? 0 : threadIdx.x / 16;
    if (r >= rows) return;  // (GROUPS == 1 only, which never synchronises)
    float ms[PER], ls[PER], m = -FLT_MAX;
    floatx4 o = {0.f, 0.f, 0.f, 0.f}, os[PER];
    const int n = (a.splits - g + GROUPS - 1) / GROUPS;  // this group's splits (may be none); indexes past them are clamped
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int64_t slot = (int64_t)min(g + i * GROUPS, a.splits - 1) * rows + r;
        const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * slot);
        os[i] = *reinterpret_cast<const floatx4*>(a.part_o + slot * kHeadDim + c);
        ms[i] = ml.x;
        ls[i] = ml.y;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) m = fmaxf(m, ms[i]);
    if constexpr (GROUPS > 1) {
        m = wave_max(m);
        if (lane == 0) wmax[wave] = m;
        __syncthreads();
        m = fmaxf(fmaxf(wmax[0], wmax[1]), fmaxf(wmax[2], wmax[3]));
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float w = i < n ? __builtin_amdgcn_exp2f(ms[i] - m) : 0.f;
        sum = fmaf(w, ls[i], sum);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = i < n ? os[i][e] : 0.f;
            o[e] = finite_f32(x) ? fmaf(w, x, o[e]) : o[e] + x;  // (a weight may be too small for fp32, not zero)
        }
    }
    if constexpr (GROUPS > 1) {  // the wave's four groups, then the four waves
#pragma unroll
        for (int d = 16; d <= 32; d *= 2) {
            sum += __shfl_xor(sum, d);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], d);
        }
        if (lane < 16) *reinterpret_cast<floatx4*>(&wout[wave][c]) = o;
        if (lane == 0) wsum[wave] = sum;
        __syncthreads();
        if (threadIdx.x >= 16) return;
        sum = wsum[0] + wsum[1] + wsum[2] + wsum[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = wout[0][c + e] + wout[1][c + e] + wout[2][c + e] + wout[3][c + e];
    }
    const float inv = 1.0f / sum;
    T* const dst = static_cast<T*>(a.out) + (r / a.heads) * a.ldo + (r % a.heads) * kHeadDim + c;
    if constexpr (BF16) *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
    else *reinterpret_cast<floatx4*>(dst) = floatx4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
}

}  // namespace

// Workgroups over the keys of one item: where the batch has few tiles, as many as bring four
// workgroups to each CU, each with two chunks at least and no more of them than pays for the join: a chunk
// takes about 0.6 us, the second launch 3 us and 0.07 us a split.  Up to eight chunks that never pays, above
// the time is least at sqrt(8 chunks) splits.
// Measured when the rule was made: one sequence of 1000 tokens, window 512, 16/4 heads, 13.4 us on two splits,
// 10.6 on four, 10.1 on eight; of 32768 tokens, 8 heads, 18.8 us on 68, 22.1 on 128; 32 sequences, window
// 4096, 16/4 heads, 32.7 us on eight, 35.8 on 16.  (A whole GPU's 256 CUs: the workspace is sized by the same rule, on the host.)
int window_splits(int64_t T, int64_t batch, int64_t heads, int64_t kv_heads, int64_t max_len, int64_t max_kv, int64_t window,
                  int64_t sinks) {
    if (T <= 0) return 1;
    const int64_t group = heads / kv_heads;
    // tiles of 64 rows that hold any; keys a tile walks: its rows' positions and window, or all
    const int64_t tiles = kv_heads * std::min((T * group + 63 * batch) / 64, batch * ((max_len * group + 63) / 64));
    const int64_t keys = std::min(max_kv, std::min(window, max_kv) + std::min(sinks, max_kv) + std::min<int64_t>(max_len, 64));
    const int64_t chunks = (keys + kWinChunk - 1) / kWinChunk;
    const int64_t most = std::min({256 * 4 / std::max<int64_t>(tiles, 1), chunks / 2, (int64_t)kWinMaxSplits});
    int64_t splits = 1;
    while (chunks > 8 && splits < most && (splits + 1) * (splits + 1) <= 8 * chunks) ++splits;
    return (int)splits;
}

size_t window_workspace(int64_t T, int64_t heads, int64_t splits) {
    return splits > 1 ? (size_t)(splits * T * heads * (kHeadDim + 2)) * sizeof(float) : 0;
}

namespace {
template <bool BF16>
void launch_join(const WinArgs& a, int splits, int64_t rows, hipStream_t s) {
    const bool few = splits <= 16;
    const int per = few ? splits : (splits + 15) / 16;
    auto* f = few ? (per <= 2 ? &k_attention_window_join<BF16, 1, 2> : per <= 4 ? &k_attention_window_join<BF16, 1, 4>
                     : per <= 8 ? &k_attention_window_join<BF16, 1, 8> : &k_attention_window_join<BF16, 1, 16>)
                  : (per <= 2 ? &k_attention_window_join<BF16, 16, 2> : per <= 4 ? &k_attention_window_join<BF16, 16, 4>
                     : per <= 8 ? &k_attention_window_join<BF16, 16, 8> : &k_attention_window_join<BF16, 16, 16>);
    hipLaunchKernelGGL(f, dim3((unsigned)(few ? (rows + 15) / 16 : rows)), dim3(256), 0, s, a);
}
}  // namespace

hipError_t launch_attention_window(const PlanView& p, int dtype, const void* q, int ldq, const void* k, int ldk,
                                   const void* v, int ldv, const WindowKeys& keys, int kv_heads, float scale, int window,
                                   int sinks, void* out, int ldo, int splits, void* workspace, hipStream_t s) {
    if (p.total_tokens == 0 || p.av_cap == 0) return hipSuccess;  // (no entries: nothing can be written)
    float* const ws = static_cast<float*>(workspace);
    const int64_t rows = (int64_t)p.total_tokens * p.heads;
    // Where every sequence's rows of a key head fill one tile (a step of single tokens), only
    // the first of each G entries holds any, and only those are launched.  Neighbouring tiles
    // of a prompt share keys and go to one XCD in runs; tiles of single tokens and splits share none and go
    // to the XCDs in turn (in runs, eight heads' splits would all be one XCD's).
    const int group = p.heads / kv_heads;
    const bool single = (int64_t)p.max_len * group <= kTile;
    // Tiles of 128 rows, whose four waves share a chunk's copies, in bf16 from groups of four on (their
    // positions span at most a chunk, else the waves wait for each other's first and last ones), where two entries
    // of a key head always make one (an odd group's would leave workgroups empty).  Us on 64 and 128
    // rows: six prompts of 1500 to 8192 tokens, 16/4 heads, window 1024 198, 190; 128 sequences to 512
    // tokens, 16/4 heads, window 128 66.0, 60.0; 256 of 17 tokens 18.2, 14.3; groups of two, 16 of 300
    // tokens, 8/4 heads 12.4, 12.8; two of 8192, 16/8 heads 593, 641.  fp32: equal.
    const bool wide = dtype == 1 && !single && splits == 1 && group >= 4 && group % 2 == 0;
    const int stride = single ? group : wide ? 2 : 1, dealt = !single && splits == 1;
    const uint32_t magic = group == 1 ? 0u : 0xffffffffu / (uint32_t)group + 1u;
    const WinArgs a{p.lengths, p.tok_off, p.av_items, p.av_cap, p.status, keys.first, keys.len, keys.rows, keys.max_len, q, k, v,
                    out, ldq, ldk, ldv, ldo, p.heads, group, magic, window, sinks, scale, p.total_tokens, splits, stride, dealt,
                    ws, ws ? ws + (int64_t)splits * rows * kHeadDim : nullptr};
    // one workgroup per entry that a plan of this capacity can hold (in rows of 2^20)
    constexpr int64_t kUnit = 8 * kStreamRun, kRow = 1 << 20;
    int64_t g = std::max<int64_t>(p.av_cap / stride, 1);
    if (dealt) g = (g + kUnit - 1) / kUnit * kUnit;  // dealing is a permutation of these
    const dim3 grid((unsigned)std::min(g, kRow), (unsigned)splits, (unsigned)((g + kRow - 1) / kRow));
    auto* f = wide ? &k_attention_window<true, 4> : dtype == 1 ? &k_attention_window<true, 2> : &k_attention_window<false, 2>;
    hipLaunchKernelGGL(f, grid, dim3((wide ? 4 : 2) * kWave), 0, s, a);
    if (splits > 1) {
        if (dtype == 1) launch_join<true>(a, splits, rows, s);
        else launch_join<false>(a, splits, rows, s);
    }
    return hipGetLastError();
}

}  // namespace rag
