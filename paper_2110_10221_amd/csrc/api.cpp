// C entry points: host-side argument validation, then kernel launches.
// Nothing here allocates device memory; every buffer comes from the caller.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../../include/ragged.h"
#include "launch.h"

namespace {

thread_local char g_last_error[512] = "";

rag_status fail(rag_status s, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
    va_end(ap);
    return s;
}

bool sync_check_enabled() {
    static const bool on = [] {
        const char* v = getenv("RAG_SYNC_CHECK");
        return v && v[0] && strcmp(v, "0") != 0;
    }();
    return on;
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

size_t elem_size(int32_t dtype) { return dtype == RAG_F32 ? 4 : 2; }

rag_status check_dtype(int32_t dtype, const char* fn) {
    if (dtype != RAG_F32 && dtype != RAG_BF16) return fail(RAG_ERR_DTYPE, "%s: dtype %d is not RAG_F32 or RAG_BF16", fn, dtype);
    return RAG_OK;
}

// After enqueueing: report a launch error; with RAG_SYNC_CHECK also wait and
// report execution errors and the plan's data-error bits.
rag_status finish(hipError_t launch_err, hipStream_t s, const int32_t* status, const char* fn) {
    if (launch_err != hipSuccess)
        return fail(RAG_ERR_HIP, "%s: launch failed: %s", fn, hipGetErrorString(launch_err));
    if (!sync_check_enabled()) return RAG_OK;
    hipError_t e = hipStreamSynchronize(s);
    if (e != hipSuccess) return fail(RAG_ERR_HIP, "%s: execution failed: %s", fn, hipGetErrorString(e));
    if (status) {
        int32_t flags = 0;
        e = hipMemcpy(&flags, status, sizeof(flags), hipMemcpyDeviceToHost);
        if (e != hipSuccess) return fail(RAG_ERR_HIP, "%s: status read failed: %s", fn, hipGetErrorString(e));
        if (flags) return fail(RAG_ERR_DATA, "%s: plan status word reports data errors 0x%x", fn, flags);
    }
    return RAG_OK;
}

// The fused attention kernel addresses a sequence's K and V rows with 32-bit
// byte offsets from the sequence's first row.
bool fused_fits(int64_t max_len, int64_t ld) { return max_len * ld * 2 <= INT32_MAX; }

// The bf16 attention operators address one item's scores (64 query rows of
// heads * max_len values) with 32-bit byte offsets.
bool op_item_fits(int64_t heads, int64_t max_len) { return 64 * heads * max_len * 2 + 64 <= INT32_MAX; }

rag_status view_plan(const rag_plan* p, rag::PlanView& v, const char* fn) {
    if (!p) return fail(RAG_ERR_ARG, "%s: plan is NULL", fn);
    if (p->batch < 1 || p->batch > RAG_MAX_BATCH)
        return fail(RAG_ERR_ARG, "%s: batch %d outside [1, %d]", fn, p->batch, RAG_MAX_BATCH);
    if (p->total_tokens < 0 || p->max_len < 0 || p->heads < 1)
        return fail(RAG_ERR_ARG, "%s: total_tokens %d, max_len %d, heads %d out of range", fn, p->total_tokens,
                    p->max_len, p->heads);
    if (p->qkt_cap < 0 || p->av_cap < 0) return fail(RAG_ERR_ARG, "%s: negative capacity", fn);
    if (p->qkt_cap > INT32_MAX || p->av_cap > INT32_MAX)
        return fail(RAG_ERR_CAPACITY, "%s: work-list capacities must stay below 2^31", fn);
    // H * max_len^2 * batch bounds every attention offset; keep it below 2^62
    if ((double)p->heads * p->max_len * p->max_len * p->batch > 4.0e18)
        return fail(RAG_ERR_SHAPE, "%s: heads * max_len^2 * batch overflows 64-bit offsets", fn);
    if (!p->lengths || !p->tok_off || !p->att_off || !p->order || !p->qkt_item_off || !p->av_item_off ||
        !p->status)
        return fail(RAG_ERR_ARG, "%s: a plan array is NULL", fn);
    if (p->total_tokens > 0 && !p->tok_seq) return fail(RAG_ERR_ARG, "%s: tok_seq is NULL", fn);
    if (p->qkt_cap > 0 && (!p->qkt_items || !aligned(p->qkt_items, 16)))
        return fail(RAG_ERR_ARG, "%s: qkt_items must be non-NULL and 16-byte aligned", fn);
    if (p->av_cap > 0 && !p->av_items) return fail(RAG_ERR_ARG, "%s: av_items is NULL", fn);
    if (!aligned(p->att_off, 8) || !aligned(p->lengths, 4) || !aligned(p->status, 4))
        return fail(RAG_ERR_ARG, "%s: misaligned plan array", fn);
    v = rag::PlanView{p->batch, p->total_tokens, p->max_len, p->heads, p->qkt_cap, p->av_cap,
                      p->lengths, p->tok_off, p->att_off, p->order, p->tok_seq, p->qkt_item_off,
                      p->av_item_off, p->qkt_items, p->av_items, p->status};
    return RAG_OK;
}

// A packed [rows, width] operand with leading dimension ld.
rag_status check_operand(const void* ptr, int64_t ld, int64_t width, int32_t dtype, size_t vec_align,
                         const char* name, const char* fn) {
    if (!ptr) return fail(RAG_ERR_ARG, "%s: %s is NULL", fn, name);
    if (ld < width) return fail(RAG_ERR_SHAPE, "%s: leading dimension of %s (%lld) < width %lld", fn, name,
                                (long long)ld, (long long)width);
    if (dtype == RAG_BF16) {
        if (!aligned(ptr, vec_align) || (ld * 2) % vec_align != 0)
            return fail(RAG_ERR_SHAPE, "%s: %s must be %zu-byte aligned with a leading dimension that keeps rows aligned",
                        fn, name, vec_align);
    } else if (!aligned(ptr, 4)) {
        return fail(RAG_ERR_SHAPE, "%s: %s must be 4-byte aligned", fn, name);
    }
    return RAG_OK;
}

bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return na && nb && pa < pb + nb && pb < pa + na;
}

size_t span_bytes(int64_t rows, int64_t ld, int64_t width, int32_t dtype) {
    return rows > 0 ? (size_t)((rows - 1) * ld + width) * elem_size(dtype) : 0;
}

int g_cu_cache[64];

}  // namespace

namespace rag {

rag_status report(rag_status status, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
    va_end(ap);
    return status;
}

int device_cu_count() {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) dev = 0;
    if (dev < 64 && g_cu_cache[dev] > 0) return g_cu_cache[dev];
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    if (dev < 64) g_cu_cache[dev] = n;
    return n;
}

}  // namespace rag

extern "C" {

const char* ragged_status_string(rag_status s) {
    switch (s) {
        case RAG_OK: return "RAG_OK";
        case RAG_ERR_ARG: return "RAG_ERR_ARG";
        case RAG_ERR_DTYPE: return "RAG_ERR_DTYPE";
        case RAG_ERR_SHAPE: return "RAG_ERR_SHAPE";
        case RAG_ERR_CAPACITY: return "RAG_ERR_CAPACITY";
        case RAG_ERR_WORKSPACE: return "RAG_ERR_WORKSPACE";
        case RAG_ERR_HIP: return "RAG_ERR_HIP";
        case RAG_ERR_DATA: return "RAG_ERR_DATA";
        default: return "RAG_ERR_UNKNOWN";
    }
}

const char* ragged_last_error(void) { return g_last_error; }

rag_status ragged_plan_capacity(int32_t batch, int32_t total_tokens, int32_t max_len, int32_t heads,
                                int64_t* qkt_cap, int64_t* av_cap) {
    const char* fn = "ragged_plan_capacity";
    if (!qkt_cap || !av_cap) return fail(RAG_ERR_ARG, "%s: output pointer is NULL", fn);
    if (batch < 1 || batch > RAG_MAX_BATCH || total_tokens < 0 || max_len < 0 || heads < 1)
        return fail(RAG_ERR_ARG, "%s: sizes out of range", fn);
    const int64_t nt_max = ((int64_t)max_len + RAG_TILE - 1) / RAG_TILE;
    const int64_t by_len = (int64_t)batch * nt_max;
    const int64_t by_tok = ((int64_t)total_tokens + (int64_t)(RAG_TILE - 1) * batch) / RAG_TILE;
    const int64_t av = (int64_t)heads * (by_len < by_tok ? by_len : by_tok);
    *av_cap = av;
    *qkt_cap = nt_max * av;
    return RAG_OK;
}

rag_status ragged_offsets(rag_plan* plan, void* stream) {
    const char* fn = "ragged_offsets";
    rag::PlanView v;
    rag_status st = view_plan(plan, v, fn);
    if (st) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_offsets(v, s), s, plan->status, fn);
}

namespace {

rag_status qkt_impl(const rag_plan* plan, const void* q, int32_t ldq, const void* k, int32_t ldk, int32_t head_dim,
                    float scale, void* scores, int64_t score_cap, int32_t dtype, void* stream, bool causal,
                    const char* fn) {
    rag::PlanView v;
    rag_status st;
    if ((st = view_plan(plan, v, fn)) || (st = check_dtype(dtype, fn))) return st;
    if (head_dim != RAG_HEAD_DIM) return fail(RAG_ERR_SHAPE, "%s: head_dim %d unsupported (only %d)", fn, head_dim, RAG_HEAD_DIM);
    const int64_t width = (int64_t)plan->heads * head_dim;
    if ((st = check_operand(q, ldq, width, dtype, 16, "q", fn)) || (st = check_operand(k, ldk, width, dtype, 16, "k", fn)))
        return st;
    if (!std::isfinite(scale)) return fail(RAG_ERR_ARG, "%s: scale is not finite", fn);
    if (!scores || score_cap < 0) return fail(RAG_ERR_ARG, "%s: scores is NULL or score_cap < 0", fn);
    if (dtype == RAG_BF16 && !op_item_fits(plan->heads, plan->max_len))
        return fail(RAG_ERR_SHAPE, "%s: 64 * heads * max_len * 2 bytes exceeds 32-bit item offsets", fn);
    if (!aligned(scores, elem_size(dtype))) return fail(RAG_ERR_ARG, "%s: scores misaligned", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_qkt(v, dtype, q, ldq, k, ldk, scale, scores, score_cap, causal, s), s, plan->status, fn);
}

rag_status softmax_impl(const rag_plan* plan, const void* scores, void* probs, int64_t score_cap, int32_t dtype,
                        void* stream, bool causal, const char* fn) {
    rag::PlanView v;
    rag_status st;
    if ((st = view_plan(plan, v, fn)) || (st = check_dtype(dtype, fn))) return st;
    if (!scores || !probs || score_cap < 0) return fail(RAG_ERR_ARG, "%s: scores/probs NULL or score_cap < 0", fn);
    // (a limit of the interface: the softmax itself addresses rows in 64 bits)
    if (dtype == RAG_BF16 && (int64_t)plan->heads * plan->max_len * 2 + 64 > INT32_MAX)
        return fail(RAG_ERR_SHAPE, "%s: heads * max_len * 2 bytes exceeds 32-bit row offsets", fn);
    if (!aligned(scores, elem_size(dtype)) || !aligned(probs, elem_size(dtype)))
        return fail(RAG_ERR_ARG, "%s: scores/probs misaligned", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_softmax(v, dtype, scores, probs, score_cap, causal, s), s, plan->status, fn);
}

rag_status attn_v_impl(const rag_plan* plan, const void* probs, int64_t score_cap, const void* vv, int32_t ldv,
                       int32_t head_dim, void* out, int32_t ldo, int32_t dtype, void* stream, bool causal,
                       const char* fn) {
    rag::PlanView v;
    rag_status st;
    if ((st = view_plan(plan, v, fn)) || (st = check_dtype(dtype, fn))) return st;
    if (head_dim != RAG_HEAD_DIM) return fail(RAG_ERR_SHAPE, "%s: head_dim %d unsupported (only %d)", fn, head_dim, RAG_HEAD_DIM);
    const int64_t width = (int64_t)plan->heads * head_dim;
    if ((st = check_operand(vv, ldv, width, dtype, 16, "v", fn)) || (st = check_operand(out, ldo, width, dtype, 16, "out", fn)))
        return st;
    if (!probs || score_cap < 0) return fail(RAG_ERR_ARG, "%s: probs is NULL or score_cap < 0", fn);
    if (!aligned(probs, elem_size(dtype))) return fail(RAG_ERR_ARG, "%s: probs misaligned", fn);
    if (dtype == RAG_BF16 && !op_item_fits(plan->heads, plan->max_len))
        return fail(RAG_ERR_SHAPE, "%s: 64 * heads * max_len * 2 bytes exceeds 32-bit item offsets", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_attn_v(v, dtype, probs, score_cap, vv, ldv, out, ldo, causal, s), s, plan->status, fn);
}

rag_status attention_impl(const rag_plan* plan, const void* q, int32_t ldq, const void* k, int32_t ldk,
                          const void* vv, int32_t ldv, int32_t head_dim, float scale, void* out, int32_t ldo,
                          int32_t dtype, void* stream, bool causal, const char* fn) {
    rag::PlanView v;
    rag_status st;
    if ((st = view_plan(plan, v, fn)) || (st = check_dtype(dtype, fn))) return st;
    if (dtype != RAG_BF16) return fail(RAG_ERR_DTYPE, "%s: the fused kernel is bf16 only", fn);
    if (head_dim != RAG_HEAD_DIM) return fail(RAG_ERR_SHAPE, "%s: head_dim %d unsupported (only %d)", fn, head_dim, RAG_HEAD_DIM);
    const int64_t width = (int64_t)plan->heads * head_dim;
    if ((st = check_operand(q, ldq, width, dtype, 16, "q", fn)) || (st = check_operand(k, ldk, width, dtype, 16, "k", fn)) ||
        (st = check_operand(vv, ldv, width, dtype, 16, "v", fn)) || (st = check_operand(out, ldo, width, dtype, 16, "out", fn)))
        return st;
    if (!std::isfinite(scale)) return fail(RAG_ERR_ARG, "%s: scale is not finite", fn);
    if (!fused_fits(plan->max_len, ldk > ldv ? ldk : ldv))
        return fail(RAG_ERR_SHAPE, "%s: max_len %d rows of leading dimension %d exceed the kernel's 32-bit offsets", fn,
                    plan->max_len, ldk > ldv ? ldk : ldv);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_fused_attention(v, dtype, q, ldq, k, ldk, vv, ldv, scale, out, ldo, causal, s), s,
                  plan->status, fn);
}

}  // namespace

rag_status ragged_qkt(const rag_plan* plan, const void* q, int32_t ldq, const void* k, int32_t ldk,
                      int32_t head_dim, float scale, void* scores, int64_t score_cap, int32_t dtype,
                      void* stream) {
    return qkt_impl(plan, q, ldq, k, ldk, head_dim, scale, scores, score_cap, dtype, stream, false, "ragged_qkt");
}

rag_status ragged_qkt_causal(const rag_plan* plan, const void* q, int32_t ldq, const void* k, int32_t ldk,
                             int32_t head_dim, float scale, void* scores, int64_t score_cap, int32_t dtype,
                             void* stream) {
    return qkt_impl(plan, q, ldq, k, ldk, head_dim, scale, scores, score_cap, dtype, stream, true,
                    "ragged_qkt_causal");
}

rag_status ragged_softmax(const rag_plan* plan, const void* scores, void* probs, int64_t score_cap, int32_t dtype,
                          void* stream) {
    return softmax_impl(plan, scores, probs, score_cap, dtype, stream, false, "ragged_softmax");
}

rag_status ragged_softmax_causal(const rag_plan* plan, const void* scores, void* probs, int64_t score_cap,
                                 int32_t dtype, void* stream) {
    return softmax_impl(plan, scores, probs, score_cap, dtype, stream, true, "ragged_softmax_causal");
}

rag_status ragged_attn_v(const rag_plan* plan, const void* probs, int64_t score_cap, const void* vv, int32_t ldv,
                         int32_t head_dim, void* out, int32_t ldo, int32_t dtype, void* stream) {
    return attn_v_impl(plan, probs, score_cap, vv, ldv, head_dim, out, ldo, dtype, stream, false, "ragged_attn_v");
}

rag_status ragged_attn_v_causal(const rag_plan* plan, const void* probs, int64_t score_cap, const void* vv,
                                int32_t ldv, int32_t head_dim, void* out, int32_t ldo, int32_t dtype,
                                void* stream) {
    return attn_v_impl(plan, probs, score_cap, vv, ldv, head_dim, out, ldo, dtype, stream, true,
                       "ragged_attn_v_causal");
}

rag_status ragged_attention(const rag_plan* plan, const void* q, int32_t ldq, const void* k, int32_t ldk,
                            const void* vv, int32_t ldv, int32_t head_dim, float scale, void* out, int32_t ldo,
                            int32_t dtype, void* stream) {
    return attention_impl(plan, q, ldq, k, ldk, vv, ldv, head_dim, scale, out, ldo, dtype, stream, false,
                          "ragged_attention");
}

rag_status ragged_attention_causal(const rag_plan* plan, const void* q, int32_t ldq, const void* k, int32_t ldk,
                                   const void* vv, int32_t ldv, int32_t head_dim, float scale, void* out,
                                   int32_t ldo, int32_t dtype, void* stream) {
    return attention_impl(plan, q, ldq, k, ldk, vv, ldv, head_dim, scale, out, ldo, dtype, stream, true,
                          "ragged_attention_causal");
}

namespace {

rag_status check_linear(const void* x, int32_t ldx, const void* w, const void* bias, const void* residual,
                        int32_t ldr, int32_t act, const void* y, int32_t ldy, int32_t T, int32_t K, int32_t N,
                        int32_t dtype, const char* fn) {
    rag_status st;
    if ((st = check_dtype(dtype, fn))) return st;
    if (T < 0 || K < 1 || N < 1) return fail(RAG_ERR_ARG, "%s: T %d, K %d, N %d out of range", fn, T, K, N);
    if (act < RAG_ACT_NONE || act > RAG_ACT_GELU_TANH) return fail(RAG_ERR_ARG, "%s: bad activation %d", fn, act);
    if (dtype == RAG_BF16 && (K % 64 != 0 || N % 64 != 0))
        return fail(RAG_ERR_SHAPE, "%s: bf16 needs K %% 64 == 0 and N %% 64 == 0 (K %d, N %d)", fn, K, N);
    if (T == 0) return RAG_OK;  // nothing is read or written
    if ((st = check_operand(x, ldx, K, dtype, 16, "x", fn)) || (st = check_operand(w, K, K, dtype, 16, "w", fn)) ||
        (st = check_operand(y, ldy, N, dtype, 16, "y", fn)))
        return st;
    if (residual && (st = check_operand(residual, ldr, N, dtype, 16, "residual", fn))) return st;
    if (bias && !aligned(bias, dtype == RAG_BF16 ? 8 : 4)) return fail(RAG_ERR_SHAPE, "%s: bias misaligned", fn);
    const size_t ys = span_bytes(T, ldy, N, dtype);
    if (ranges_overlap(y, ys, x, span_bytes(T, ldx, K, dtype)) ||
        ranges_overlap(y, ys, w, span_bytes(N, K, K, dtype)))
        return fail(RAG_ERR_ARG, "%s: y overlaps x or w", fn);
    if (residual && residual != y && ranges_overlap(y, ys, residual, span_bytes(T, ldr, N, dtype)))
        return fail(RAG_ERR_ARG, "%s: residual partially overlaps y", fn);
    if (residual == y && ldr != ldy) return fail(RAG_ERR_ARG, "%s: in-place residual needs ldr == ldy", fn);
    return RAG_OK;
}

rag_status check_layernorm(const void* x, int32_t ldx, const void* g, const void* b, const void* y, int32_t ldy,
                           int32_t T, int32_t d, int32_t dtype, const char* fn) {
    rag_status st;
    if ((st = check_dtype(dtype, fn))) return st;
    if (T < 0 || d < 1) return fail(RAG_ERR_ARG, "%s: T %d, d %d out of range", fn, T, d);
    const int per = dtype == RAG_BF16 ? 8 : 4;
    if (d % per != 0 || d > 4096) return fail(RAG_ERR_SHAPE, "%s: d %d must be a multiple of %d and <= 4096", fn, d, per);
    if (T == 0) return RAG_OK;  // nothing is read or written
    if ((st = check_operand(x, ldx, d, dtype, 16, "x", fn)) || (st = check_operand(y, ldy, d, dtype, 16, "y", fn)))
        return st;
    if (dtype == RAG_F32 && (!aligned(x, 16) || !aligned(y, 16) || ldx % 4 || ldy % 4))
        return fail(RAG_ERR_SHAPE, "%s: fp32 rows must be 16-byte aligned", fn);
    if (!g || !b || !aligned(g, 16) || !aligned(b, 16)) return fail(RAG_ERR_ARG, "%s: gamma/beta NULL or misaligned", fn);
    if (x != y && ranges_overlap(y, span_bytes(T, ldy, d, dtype), x, span_bytes(T, ldx, d, dtype)))
        return fail(RAG_ERR_ARG, "%s: y partially overlaps x", fn);
    if (x == y && ldx != ldy) return fail(RAG_ERR_ARG, "%s: in-place use needs ldx == ldy", fn);
    return RAG_OK;
}

}  // namespace

rag_status packed_linear(const void* x, int32_t ldx, const void* w, const void* bias, const void* residual,
                         int32_t ldr, int32_t act, void* y, int32_t ldy, int32_t T, int32_t K, int32_t N,
                         int32_t dtype, void* stream) {
    const char* fn = "packed_linear";
    rag_status st = check_linear(x, ldx, w, bias, residual, ldr, act, y, ldy, T, K, N, dtype, fn);
    if (st) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_linear(dtype, x, ldx, w, bias, residual, ldr, act, y, ldy, T, K, N, s), s, nullptr, fn);
}

rag_status packed_layernorm(const void* x, int32_t ldx, const void* gamma, const void* beta, float eps, void* y,
                            int32_t ldy, int32_t T, int32_t d, int32_t dtype, void* stream) {
    const char* fn = "packed_layernorm";
    rag_status st = check_layernorm(x, ldx, gamma, beta, y, ldy, T, d, dtype, fn);
    if (st) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_layernorm(dtype, x, ldx, gamma, beta, eps, y, ldy, T, d, s), s, nullptr, fn);
}

namespace {

constexpr size_t kAlign = 256;
size_t round_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

// The fused attention kernel exists for bf16 (and sequences whose K / V rows its
// 32-bit offsets reach); other layers run the three attention operators over a
// materialised score buffer.  The layer's Q, K and V are column blocks of one
// [T, 3d] buffer.
bool unfused_attention(int32_t dtype, int32_t flags, int64_t max_len, int64_t d) {
    return (flags & RAG_LAYER_UNFUSED_ATTENTION) || dtype == RAG_F32 || !fused_fits(max_len, 3 * d);
}

struct LayerBuffers {
    size_t qkvf, act_a, h1o, scores, total;
};

LayerBuffers layer_buffers(int64_t T, int64_t max_len, int64_t d, int64_t H, int64_t d_ff, int32_t dtype,
                           int32_t flags) {
    const size_t es = elem_size(dtype);
    LayerBuffers lb{};
    lb.qkvf = round_up((size_t)T * (size_t)(3 * d > d_ff ? 3 * d : d_ff) * es);  // QKV, later FF1 output
    lb.act_a = round_up((size_t)T * d * es);                                     // Y1, later Y2
    lb.h1o = round_up((size_t)T * d * es);                                       // attention output, later H1
    lb.scores = unfused_attention(dtype, flags, max_len, d) ? round_up((size_t)H * T * max_len * es) : 0;
    lb.total = lb.qkvf + lb.act_a + lb.h1o + lb.scores;
    return lb;
}

}  // namespace

rag_status encoder_layer_workspace(int32_t total_tokens, int32_t max_len, int32_t d_model, int32_t heads,
                                   int32_t d_ff, int32_t dtype, int32_t flags, size_t* bytes) {
    const char* fn = "encoder_layer_workspace";
    rag_status st;
    if ((st = check_dtype(dtype, fn))) return st;
    if (!bytes) return fail(RAG_ERR_ARG, "%s: bytes is NULL", fn);
    if (total_tokens < 0 || max_len < 0 || d_model < 1 || heads < 1 || d_ff < 1)
        return fail(RAG_ERR_ARG, "%s: sizes out of range", fn);
    *bytes = layer_buffers(total_tokens, max_len, d_model, heads, d_ff, dtype, flags).total;
    return RAG_OK;
}

rag_status encoder_layer(const rag_plan* plan, const void* x, void* y, int32_t d_model, int32_t heads,
                         int32_t head_dim, int32_t d_ff, float ln_eps, int32_t act, int32_t flags,
                         const rag_layer_weights* w, void* workspace, size_t workspace_bytes, int32_t dtype,
                         void* stream, void* const* events) {
    const char* fn = "encoder_layer";
    rag::PlanView v;
    rag_status st;
    if ((st = view_plan(plan, v, fn)) || (st = check_dtype(dtype, fn))) return st;
    if (!w) return fail(RAG_ERR_ARG, "%s: weights is NULL", fn);
    if (heads != plan->heads) return fail(RAG_ERR_SHAPE, "%s: heads %d differs from the plan's %d", fn, heads, plan->heads);
    if (head_dim != RAG_HEAD_DIM) return fail(RAG_ERR_SHAPE, "%s: head_dim %d unsupported (only %d)", fn, head_dim, RAG_HEAD_DIM);
    if (d_model != heads * head_dim) return fail(RAG_ERR_SHAPE, "%s: d_model %d != heads * head_dim", fn, d_model);
    if (flags & ~(RAG_LAYER_UNFUSED_ATTENTION | RAG_LAYER_CAUSAL | RAG_LAYER_BUILD_PLAN))
        return fail(RAG_ERR_ARG, "%s: unknown flags 0x%x", fn, flags);
    const int T = plan->total_tokens, d = d_model;
    if (dtype == RAG_BF16 && unfused_attention(dtype, flags, plan->max_len, d) && !op_item_fits(heads, plan->max_len))
        return fail(RAG_ERR_SHAPE, "%s: 64 * heads * max_len * 2 bytes exceeds 32-bit item offsets", fn);
    const LayerBuffers lb = layer_buffers(T, plan->max_len, d, heads, d_ff, dtype, flags);
    if (!workspace || workspace_bytes < lb.total)
        return fail(RAG_ERR_WORKSPACE, "%s: workspace of %zu bytes given, %zu needed", fn, workspace_bytes, lb.total);
    if (!aligned(workspace, kAlign)) return fail(RAG_ERR_WORKSPACE, "%s: workspace must be %zu-byte aligned", fn, kAlign);
    char* ws = static_cast<char*>(workspace);
    void* qkv = ws;                      // [T, 3d], later F [T, d_ff]
    void* act_a = ws + lb.qkvf;          // Y1, later Y2
    void* h1o = ws + lb.qkvf + lb.act_a;  // attention output O, later H1
    void* scores = ws + lb.qkvf + lb.act_a + lb.h1o;
    const size_t es = elem_size(dtype);
    const char* qkvc = static_cast<const char*>(qkv);
    // every token-wise step is validated up front, so nothing is launched unless all are valid
    if ((st = check_linear(x, d, w->w_qkv, w->b_qkv, nullptr, 0, RAG_ACT_NONE, qkv, 3 * d, T, d, 3 * d, dtype, fn)) ||
        (st = check_linear(h1o, d, w->w_o, w->b_o, x, d, RAG_ACT_NONE, act_a, d, T, d, d, dtype, fn)) ||
        (st = check_layernorm(act_a, d, w->ln1_g, w->ln1_b, h1o, d, T, d, dtype, fn)) ||
        (st = check_linear(h1o, d, w->w_ff1, w->b_ff1, nullptr, 0, act, qkv, d_ff, T, d, d_ff, dtype, fn)) ||
        (st = check_linear(qkv, d_ff, w->w_ff2, w->b_ff2, h1o, d, RAG_ACT_NONE, act_a, d, T, d_ff, d, dtype, fn)) ||
        (st = check_layernorm(act_a, d, w->ln2_g, w->ln2_b, y, d, T, d, dtype, fn)))
        return st;
    if (ranges_overlap(x, span_bytes(T, d, d, dtype), y, span_bytes(T, d, d, dtype)))
        return fail(RAG_ERR_ARG, "%s: x and y overlap", fn);
    if (ranges_overlap(ws, lb.total, x, span_bytes(T, d, d, dtype)) ||
        ranges_overlap(ws, lb.total, y, span_bytes(T, d, d, dtype)))
        return fail(RAG_ERR_ARG, "%s: workspace overlaps x or y", fn);

    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    auto mark = [&](int k) {
        if (events && e == hipSuccess) e = hipEventRecord(static_cast<hipEvent_t>(events[k]), s);
    };
    auto run = [&](hipError_t r) {
        if (e == hipSuccess) e = r;
    };
    const float scale = 1.0f / sqrtf((float)head_dim);
    const bool causal = (flags & RAG_LAYER_CAUSAL) != 0;
    mark(0);
    run(rag::launch_linear(dtype, x, d, w->w_qkv, w->b_qkv, nullptr, 0, RAG_ACT_NONE, qkv, 3 * d, T, d, 3 * d, s,
                           (flags & RAG_LAYER_BUILD_PLAN) ? &v : nullptr));
    mark(1);
    if (unfused_attention(dtype, flags, plan->max_len, d)) {
        const int64_t cap = (int64_t)(lb.scores / es);
        run(rag::launch_qkt(v, dtype, qkvc, 3 * d, qkvc + es * d, 3 * d, scale, scores, cap, causal, s));
        mark(2);
        run(rag::launch_softmax(v, dtype, scores, scores, cap, causal, s));
        mark(3);
        run(rag::launch_attn_v(v, dtype, scores, cap, qkvc + 2 * es * d, 3 * d, h1o, d, causal, s));
    } else {
        mark(2);
        mark(3);
        run(rag::launch_fused_attention(v, dtype, qkvc, 3 * d, qkvc + es * d, 3 * d, qkvc + 2 * es * d, 3 * d, scale,
                                        h1o, d, causal, s));
    }
    mark(4);
    run(rag::launch_linear(dtype, h1o, d, w->w_o, w->b_o, x, d, RAG_ACT_NONE, act_a, d, T, d, d, s));
    mark(5);
    run(rag::launch_layernorm(dtype, act_a, d, w->ln1_g, w->ln1_b, ln_eps, h1o, d, T, d, s));
    mark(6);
    run(rag::launch_linear(dtype, h1o, d, w->w_ff1, w->b_ff1, nullptr, 0, act, qkv, d_ff, T, d, d_ff, s));
    mark(7);
    run(rag::launch_linear(dtype, qkv, d_ff, w->w_ff2, w->b_ff2, h1o, d, RAG_ACT_NONE, act_a, d, T, d_ff, d, s));
    mark(8);
    run(rag::launch_layernorm(dtype, act_a, d, w->ln2_g, w->ln2_b, ln_eps, y, d, T, d, s));
    mark(9);
    return finish(e, s, plan->status, fn);
}

namespace {

rag_status view_vgemm_plan(const rag_vgemm_plan* p, rag::VgemmView& v, const char* fn) {
    if (!p) return fail(RAG_ERR_ARG, "%s: plan is NULL", fn);
    if (p->batch < 1 || p->batch > RAG_VGEMM_MAX_BATCH)
        return fail(RAG_ERR_ARG, "%s: batch %d outside [1, %d]", fn, p->batch, RAG_VGEMM_MAX_BATCH);
    if (p->tile_cap < 0) return fail(RAG_ERR_ARG, "%s: negative tile_cap", fn);
    if (p->tile_cap > RAG_VGEMM_MAX_TILES)
        return fail(RAG_ERR_CAPACITY, "%s: tile_cap %lld exceeds %d", fn, (long long)p->tile_cap, RAG_VGEMM_MAX_TILES);
    if (!p->dims || !p->a_off || !p->b_off || !p->c_off || !p->order || !p->tile_off || !p->status)
        return fail(RAG_ERR_ARG, "%s: a plan array is NULL", fn);
    if (p->tile_cap > 0 && (!p->tile_items || !aligned(p->tile_items, 16)))
        return fail(RAG_ERR_ARG, "%s: tile_items must be non-NULL and 16-byte aligned", fn);
    if (!aligned(p->dims, 4) || !aligned(p->a_off, 8) || !aligned(p->b_off, 8) || !aligned(p->c_off, 8) ||
        !aligned(p->order, 4) || !aligned(p->tile_off, 8) || !aligned(p->status, 4))
        return fail(RAG_ERR_ARG, "%s: misaligned plan array", fn);
    v = rag::VgemmView{p->batch, p->tile_cap, p->dims, p->a_off, p->b_off, p->c_off, p->order,
                       p->tile_off, p->tile_items, p->status};
    return RAG_OK;
}

}  // namespace

rag_status vgemm_plan_capacity(int32_t batch, int32_t max_m, int32_t max_n, int64_t* tile_cap) {
    const char* fn = "vgemm_plan_capacity";
    if (!tile_cap) return fail(RAG_ERR_ARG, "%s: output pointer is NULL", fn);
    if (batch < 1 || batch > RAG_VGEMM_MAX_BATCH || max_m < 0 || max_n < 0 || max_m > RAG_VGEMM_MAX_DIM ||
        max_n > RAG_VGEMM_MAX_DIM)
        return fail(RAG_ERR_ARG, "%s: sizes out of range", fn);
    *tile_cap = (int64_t)batch * ((max_m + RAG_VGEMM_TILE_M - 1) / RAG_VGEMM_TILE_M) *
                ((max_n + RAG_VGEMM_TILE_N - 1) / RAG_VGEMM_TILE_N);
    return RAG_OK;
}

rag_status vgemm_tile_count(int32_t batch, const int32_t* dims, int64_t* tiles) {
    const char* fn = "vgemm_tile_count";
    if (!dims || !tiles) return fail(RAG_ERR_ARG, "%s: dims or tiles is NULL", fn);
    if (batch < 1 || batch > RAG_VGEMM_MAX_BATCH)
        return fail(RAG_ERR_ARG, "%s: batch %d outside [1, %d]", fn, batch, RAG_VGEMM_MAX_BATCH);
    int64_t n = 0;
    for (int32_t p = 0; p < batch; ++p) {
        const int32_t m = dims[3 * p], nn = dims[3 * p + 1], k = dims[3 * p + 2];
        if (m < 0 || nn < 0 || k < 0 || m > RAG_VGEMM_MAX_DIM || nn > RAG_VGEMM_MAX_DIM || k > RAG_VGEMM_MAX_DIM)
            return fail(RAG_ERR_ARG, "%s: problem %d has sizes (%d, %d, %d) outside [0, %d]", fn, p, m, nn, k,
                        RAG_VGEMM_MAX_DIM);
        n += (int64_t)((m + RAG_VGEMM_TILE_M - 1) / RAG_VGEMM_TILE_M) * ((nn + RAG_VGEMM_TILE_N - 1) / RAG_VGEMM_TILE_N);
    }
    *tiles = n;
    return RAG_OK;
}

rag_status vgemm_offsets(rag_vgemm_plan* plan, void* stream) {
    const char* fn = "vgemm_offsets";
    rag::VgemmView v;
    rag_status st = view_vgemm_plan(plan, v, fn);
    if (st) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_vgemm_offsets(v, s), s, plan->status, fn);
}

rag_status ragged_vgemm(const rag_vgemm_plan* plan, const void* a, int64_t a_cap, const void* b, int64_t b_cap,
                        void* c, int64_t c_cap, int32_t dtype, void* stream) {
    const char* fn = "ragged_vgemm";
    rag::VgemmView v;
    rag_status st;
    if ((st = view_vgemm_plan(plan, v, fn)) || (st = check_dtype(dtype, fn))) return st;
    if (a_cap < 0 || b_cap < 0 || c_cap < 0) return fail(RAG_ERR_ARG, "%s: negative operand capacity", fn);
    if ((a_cap && !a) || (b_cap && !b) || (c_cap && !c)) return fail(RAG_ERR_ARG, "%s: a, b or c is NULL", fn);
    const size_t align = dtype == RAG_BF16 ? 16 : 4;
    if (!aligned(a, align) || !aligned(b, align) || !aligned(c, align))
        return fail(RAG_ERR_SHAPE, "%s: a, b and c must be %zu-byte aligned", fn, align);
    const size_t es = elem_size(dtype);
    if (ranges_overlap(c, c_cap * es, a, a_cap * es) || ranges_overlap(c, c_cap * es, b, b_cap * es))
        return fail(RAG_ERR_ARG, "%s: c overlaps a or b", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_vgemm(v, dtype, a, a_cap, b, b_cap, c, c_cap, s), s, plan->status, fn);
}

rag_status ragged_trmm(const void* l, int32_t ldl, const void* b, int32_t ldb, void* c, int32_t ldc, int32_t n,
                       int32_t m, int32_t dtype, void* stream) {
    const char* fn = "ragged_trmm";
    rag_status st;
    if ((st = check_dtype(dtype, fn))) return st;
    if (n < 0 || m < 0) return fail(RAG_ERR_ARG, "%s: negative size (n %d, m %d)", fn, n, m);
    if (n == 0 || m == 0) return RAG_OK;
    if ((st = check_operand(l, ldl, n, dtype, 16, "L", fn)) || (st = check_operand(b, ldb, m, dtype, 16, "B", fn)) ||
        (st = check_operand(c, ldc, m, dtype, 16, "C", fn)))
        return st;
    if (dtype == RAG_BF16) {
        if (m % 8 != 0) return fail(RAG_ERR_SHAPE, "%s: bf16 needs m %% 8 == 0 (m = %d)", fn, m);
        // 32-bit buffer offsets: B rows up to n rounded to 64, 128-row panels of L
        if ((int64_t)(n + 64) * ldb >= (int64_t)1 << 30 || ldl >= 1 << 23)
            return fail(RAG_ERR_SHAPE, "%s: bf16 needs (n + 64) * ldb < 2^30 and ldl < 2^23", fn);
    }
    const size_t lc = span_bytes(n, ldc, m, dtype);
    if (ranges_overlap(c, lc, l, span_bytes(n, ldl, n, dtype)) || ranges_overlap(c, lc, b, span_bytes(n, ldb, m, dtype)))
        return fail(RAG_ERR_ARG, "%s: C overlaps L or B", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_trmm(dtype, l, ldl, b, ldb, c, ldc, n, m, s), s, nullptr, fn);
}

namespace {

constexpr int32_t kMaxRows = 1 << 24;  // rows
constexpr int32_t kMaxKeys = 1 << 30;  // keys of a sequence: position arithmetic stays in 32 bits

// Rows read and written in 16-byte chunks in either type.
rag_status check_rows(const void* ptr, int64_t ld, int64_t width, int32_t dtype, const char* name, const char* fn) {
    const rag_status st = check_operand(ptr, ld, width, dtype, 16, name, fn);
    if (st) return st;
    if (!aligned(ptr, 16) || ld * (int64_t)elem_size(dtype) % 16 != 0)
        return fail(RAG_ERR_SHAPE, "%s: %s needs 16-byte aligned rows", fn, name);
    return RAG_OK;
}

size_t span8(int64_t rows, int64_t ld, int64_t width) { return rows > 0 ? (size_t)((rows - 1) * ld + width) : 0; }

// An output in 8-bit rows of per-element chunks of E values.
rag_status check_q(const int8_t* q, int64_t ldq, const float* scale, int64_t d, int E, const char* fn) {
    if (!q || !scale) return fail(RAG_ERR_ARG, "%s: q and its scale go together", fn);
    if (ldq < d) return fail(RAG_ERR_SHAPE, "%s: leading dimension of q (%lld) < width %lld", fn, (long long)ldq, (long long)d);
    if (!aligned(q, E) || ldq % E != 0)
        return fail(RAG_ERR_SHAPE, "%s: q must be %d-byte aligned with a leading dimension that is a multiple of %d", fn, E, E);
    if (!aligned(scale, 4)) return fail(RAG_ERR_SHAPE, "%s: scale misaligned", fn);
    return RAG_OK;
}

rag_status check_norm_sizes(int32_t T, int32_t d, int32_t dtype, const char* fn) {
    const rag_status st = check_dtype(dtype, fn);
    if (st) return st;
    if (T < 0 || T > kMaxRows || d < 1) return fail(RAG_ERR_ARG, "%s: T %d, d %d out of range", fn, T, d);
    const int E = dtype == RAG_BF16 ? 8 : 4;
    if (d % E != 0 || d > RAG_NORM_MAX_DIM)
        return fail(RAG_ERR_SHAPE, "%s: d %d must be a multiple of %d and <= %d", fn, d, E, RAG_NORM_MAX_DIM);
    return RAG_OK;
}

struct Span {
    const void* p;
    size_t n;
    int64_t ld;
};

// Outputs against inputs they may equal exactly (same address and row stride) and against
// everything else.
bool clash(const Span& out, const Span& in) {
    if (!out.p || !in.p || !ranges_overlap(out.p, out.n, in.p, in.n)) return false;
    return !(out.p == in.p && out.ld == in.ld);
}

}  // namespace

rag_status packed_rmsnorm(const void* x, int32_t ldx, const void* residual, int32_t ldr, const void* gamma, float eps,
                          void* sum, int32_t lds, void* y, int32_t ldy, int8_t* q, int32_t ldq, float* q_scale,
                          int32_t T, int32_t d, int32_t dtype, void* stream) {
    const char* fn = "packed_rmsnorm";
    rag_status st;
    if ((st = check_norm_sizes(T, d, dtype, fn))) return st;
    if (!(eps > 0.f) || !std::isfinite(eps)) return fail(RAG_ERR_ARG, "%s: eps must be positive and finite", fn);
    if (T == 0) return RAG_OK;  // nothing is read or written
    if ((st = check_rows(x, ldx, d, dtype, "x", fn))) return st;
    if (residual && (st = check_rows(residual, ldr, d, dtype, "residual", fn))) return st;
    if (!gamma || !aligned(gamma, 16)) return fail(RAG_ERR_ARG, "%s: gamma NULL or misaligned", fn);
    if (!y && !q) return fail(RAG_ERR_ARG, "%s: neither y nor q is given", fn);
    if (sum && (st = check_rows(sum, lds, d, dtype, "sum", fn))) return st;
    if (y && (st = check_rows(y, ldy, d, dtype, "y", fn))) return st;
    if ((q || q_scale) && (st = check_q(q, ldq, q_scale, d, dtype == RAG_BF16 ? 8 : 4, fn))) return st;
    const Span sx{x, span_bytes(T, ldx, d, dtype), ldx}, sr{residual, span_bytes(T, ldr, d, dtype), ldr};
    const Span sg{gamma, d * elem_size(dtype), 0};
    const Span ss{sum, span_bytes(T, lds, d, dtype), lds}, sy{y, span_bytes(T, ldy, d, dtype), ldy};
    const Span sq{q, q ? span8(T, ldq, d) : 0, -1}, sc{q_scale, (size_t)T * 4, -2};
    if (clash(ss, sx) || clash(ss, sr) || clash(sy, sx) || clash(sy, sr))
        return fail(RAG_ERR_ARG, "%s: sum or y partially overlaps x or residual", fn);
    const Span outs[4] = {ss, sy, sq, sc};
    for (int i = 0; i < 4; ++i) {
        if (outs[i].p && ranges_overlap(outs[i].p, outs[i].n, sg.p, sg.n)) return fail(RAG_ERR_ARG, "%s: an output overlaps gamma", fn);
        for (int j = i + 1; j < 4; ++j)
            if (outs[i].p && outs[j].p && ranges_overlap(outs[i].p, outs[i].n, outs[j].p, outs[j].n))
                return fail(RAG_ERR_ARG, "%s: two outputs overlap", fn);
    }
    if (clash(sq, sx) || clash(sq, sr) || clash(sc, sx) || clash(sc, sr))
        return fail(RAG_ERR_ARG, "%s: q or its scale overlaps x or residual", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_rmsnorm(dtype, x, ldx, residual, ldr, gamma, eps, sum, lds, y, ldy, q, ldq, q_scale, T, d, s),
                  s, nullptr, fn);
}

rag_status packed_quantize_i8(const void* x, int32_t ldx, int8_t* q, int32_t ldq, float* scale, int32_t T, int32_t d,
                              int32_t dtype, void* stream) {
    const char* fn = "packed_quantize_i8";
    rag_status st;
    if ((st = check_norm_sizes(T, d, dtype, fn))) return st;
    if (T == 0) return RAG_OK;
    if ((st = check_rows(x, ldx, d, dtype, "x", fn)) || (st = check_q(q, ldq, scale, d, dtype == RAG_BF16 ? 8 : 4, fn)))
        return st;
    const Span sx{x, span_bytes(T, ldx, d, dtype), ldx};
    const Span sq{q, span8(T, ldq, d), -1}, sc{scale, (size_t)T * 4, -2};
    if (clash(sq, sx) || clash(sc, sx) || ranges_overlap(sq.p, sq.n, sc.p, sc.n))
        return fail(RAG_ERR_ARG, "%s: x, q and scale overlap", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_quantize_i8(dtype, x, ldx, q, ldq, scale, T, d, s), s, nullptr, fn);
}

rag_status rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, int32_t orig_len,
                              double beta_fast, double beta_slow, double* inv_freq, double* amplitude) {
    const char* fn = "rotary_frequencies";
    if (!inv_freq || !amplitude) return fail(RAG_ERR_ARG, "%s: output pointer is NULL", fn);
    if (rot_dim < 2 || rot_dim > RAG_ROTARY_MAX_DIM || rot_dim % 2 != 0)
        return fail(RAG_ERR_SHAPE, "%s: rot_dim %d must be even and in [2, %d]", fn, rot_dim, RAG_ROTARY_MAX_DIM);
    if (!(base > 1.0) || !std::isfinite(base)) return fail(RAG_ERR_ARG, "%s: base must be finite and above 1", fn);
    if (scaling < RAG_ROTARY_PLAIN || scaling > RAG_ROTARY_YARN) return fail(RAG_ERR_ARG, "%s: bad scaling %d", fn, scaling);
    if (scaling != RAG_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor)))
        return fail(RAG_ERR_ARG, "%s: factor must be finite and at least 1", fn);
    if (scaling == RAG_ROTARY_YARN &&
        (orig_len < 1 || !(beta_slow > 0.0) || !(beta_fast >= beta_slow) || !std::isfinite(beta_fast)))
        return fail(RAG_ERR_ARG, "%s: needs orig_len >= 1 and beta_fast >= beta_slow > 0", fn);
    if (scaling == RAG_ROTARY_NTK && rot_dim > 2) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
    if (!std::isfinite(base)) return fail(RAG_ERR_ARG, "%s: the scaled base is not finite", fn);
    *amplitude = 1.0;
    double lo = 0.0, hi = 0.0;
    if (scaling == RAG_ROTARY_YARN) {
        // pair i turns orig_len * base^(-2i / rot_dim) / (2 pi) times over the original length;
        // the pairs that turn beta times, as real numbers
        const double two_pi = 6.283185307179586477, per = 0.5 * rot_dim / std::log(base);
        lo = std::max(std::floor(per * std::log(orig_len / (beta_fast * two_pi))), 0.0);
        hi = std::min(std::ceil(per * std::log(orig_len / (beta_slow * two_pi))), rot_dim - 1.0);
        *amplitude = 0.1 * std::log(factor) + 1.0;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        inv_freq[i] = scaling == RAG_ROTARY_LINEAR ? f / factor : f;
        if (scaling == RAG_ROTARY_YARN) {
            const double ramp = std::min(std::max((i - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
            inv_freq[i] = f * (1.0 - ramp) + f / factor * ramp;
        }
    }
    return RAG_OK;
}

rag_status packed_rotary(const rag_plan* plan, const void* x, int32_t ldx, void* y, int32_t ldy, int32_t heads,
                         int32_t head_dim, int32_t rot_dim, int32_t layout, const double* inv_freq, float amplitude,
                         const int32_t* pos_start, int32_t dtype, void* stream) {
    const char* fn = "packed_rotary";
    rag::PlanView v;
    rag_status st;
    if ((st = view_plan(plan, v, fn)) || (st = check_dtype(dtype, fn))) return st;
    if (heads < 1 || plan->total_tokens > kMaxRows)
        return fail(RAG_ERR_ARG, "%s: heads %d or total_tokens %d out of range", fn, heads, plan->total_tokens);
    if (layout < 0 || layout > (RAG_ROTARY_INTERLEAVED | RAG_ROTARY_INVERSE)) return fail(RAG_ERR_ARG, "%s: bad layout %d", fn, layout);
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > head_dim || head_dim > RAG_ROTARY_MAX_DIM)
        return fail(RAG_ERR_SHAPE, "%s: rot_dim %d must be even and in [2, head_dim], head_dim %d at most %d", fn, rot_dim,
                    head_dim, RAG_ROTARY_MAX_DIM);
    if ((int64_t)heads * head_dim > (1 << 26)) return fail(RAG_ERR_SHAPE, "%s: %d heads of %d are too wide", fn, heads, head_dim);
    if (!std::isfinite(amplitude)) return fail(RAG_ERR_ARG, "%s: amplitude is not finite", fn);
    if (plan->total_tokens == 0) return RAG_OK;  // nothing is read or written
    const int64_t width = (int64_t)heads * head_dim, es = (int64_t)elem_size(dtype);
    if ((st = check_operand(x, ldx, width, dtype, es, "x", fn)) || (st = check_operand(y, ldy, width, dtype, es, "y", fn)))
        return st;
    if (!inv_freq || !aligned(inv_freq, 8)) return fail(RAG_ERR_ARG, "%s: inv_freq NULL or misaligned", fn);
    if (!aligned(pos_start, 4)) return fail(RAG_ERR_ARG, "%s: pos_start misaligned", fn);
    const int64_t T = plan->total_tokens;
    const Span sx{x, span_bytes(T, ldx, width, dtype), ldx}, sy{y, span_bytes(T, ldy, width, dtype), ldy};
    if (clash(sy, sx)) return fail(RAG_ERR_ARG, "%s: y partially overlaps x", fn);
    if (ranges_overlap(sy.p, sy.n, inv_freq, 4 * rot_dim) ||
        (pos_start && ranges_overlap(sy.p, sy.n, pos_start, 4 * (size_t)plan->batch)))
        return fail(RAG_ERR_ARG, "%s: y overlaps inv_freq or pos_start", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_rotary(v, dtype, x, ldx, y, ldy, heads, head_dim, rot_dim, !(layout & RAG_ROTARY_INTERLEAVED),
                                     (layout & RAG_ROTARY_INVERSE) != 0, inv_freq, amplitude, pos_start, s),
                  s, plan->status, fn);
}

rag_status packed_linear_i8(const int8_t* x, int32_t ldx, const float* x_scale, const int8_t* w, const float* w_scale,
                            const void* bias, const void* residual, int32_t ldr, int32_t act, void* y, int32_t ldy,
                            int32_t T, int32_t K, int32_t N, int32_t dtype, void* stream) {
    const char* fn = "packed_linear_i8";
    rag_status st;
    if ((st = check_dtype(dtype, fn))) return st;
    if (T < 0 || T > kMaxRows || K < 1 || N < 1 || N > kMaxRows)
        return fail(RAG_ERR_ARG, "%s: T %d, K %d, N %d out of range", fn, T, K, N);
    if (act < RAG_ACT_NONE || act > RAG_ACT_GELU_TANH) return fail(RAG_ERR_ARG, "%s: bad activation %d", fn, act);
    if (K % 16 != 0 || K > RAG_I8_MAX_K || N % 8 != 0)
        return fail(RAG_ERR_SHAPE, "%s: needs K %% 16 == 0, K <= %d and N %% 8 == 0 (K %d, N %d)", fn, RAG_I8_MAX_K, K, N);
    if (T == 0) return RAG_OK;  // nothing is read or written
    if (!x || !w || !x_scale || !w_scale) return fail(RAG_ERR_ARG, "%s: an operand or its scale is NULL", fn);
    if (ldx < K || ldx >= (1 << 22) || ldx % 16 != 0 || !aligned(x, 16) || !aligned(w, 16))
        return fail(RAG_ERR_SHAPE, "%s: x and w must be 16-byte aligned, ldx %d a multiple of 16 in [K, 2^22)", fn, ldx);
    if (!aligned(x_scale, 4) || !aligned(w_scale, 16))
        return fail(RAG_ERR_SHAPE, "%s: x_scale must be 4-byte and w_scale 16-byte aligned", fn);
    if ((st = check_rows(y, ldy, N, dtype, "y", fn))) return st;
    if (residual && (st = check_rows(residual, ldr, N, dtype, "residual", fn))) return st;
    if (bias && !aligned(bias, 16)) return fail(RAG_ERR_SHAPE, "%s: bias misaligned", fn);
    const Span sy{y, span_bytes(T, ldy, N, dtype), ldy};
    const Span in[6] = {{x, span8(T, ldx, K), -1}, {w, span8(N, K, K), -1}, {x_scale, (size_t)T * 4, -1},
                        {w_scale, (size_t)N * 4, -1}, {bias, (size_t)N * elem_size(dtype), -1},
                        {residual, span_bytes(T, ldr, N, dtype), ldr}};
    for (const Span& i : in)
        if (clash(sy, i)) return fail(RAG_ERR_ARG, "%s: y overlaps an input (only residual may equal it, with its ld)", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_linear_i8(dtype, x, ldx, x_scale, w, w_scale, bias, residual, ldr, act, y, ldy, T, K, N, s), s,
                  nullptr, fn);
}

namespace {

constexpr int32_t kWindowMaxLd = 1 << 22;  // 32 rows of a chunk in 32-bit byte offsets

rag_status check_window(const rag_plan* plan, rag::PlanView& v, int32_t max_kv_len, int32_t kv_heads, int32_t window,
                        int32_t sinks, int32_t dtype, const char* fn) {
    rag_status st;
    if ((st = view_plan(plan, v, fn)) || (st = check_dtype(dtype, fn))) return st;
    if (kv_heads < 1 || plan->heads % kv_heads != 0)
        return fail(RAG_ERR_SHAPE, "%s: %d heads are not a multiple of %d key heads", fn, plan->heads, kv_heads);
    if (plan->heads > 32768) return fail(RAG_ERR_SHAPE, "%s: more than 32768 heads", fn);
    if (window < 0 || sinks < 0 || max_kv_len < 0 || max_kv_len > kMaxKeys || plan->total_tokens > kMaxRows)
        return fail(RAG_ERR_ARG, "%s: window %d, sinks %d, max_kv_len %d or total_tokens %d out of range", fn, window, sinks,
                    max_kv_len, plan->total_tokens);
    if (((int64_t)plan->total_tokens + RAG_TILE) * (plan->heads / kv_heads) > INT32_MAX)
        return fail(RAG_ERR_SHAPE, "%s: tokens * heads per key head exceed 2^31 - 1", fn);
    return RAG_OK;
}

rag_status window_impl(const rag_plan* plan, const void* q, int32_t ldq, const void* k, int32_t ldk, const void* vv,
                       int32_t ldv, const rag::WindowKeys& keys, int32_t kv_heads, int32_t head_dim, float scale,
                       int32_t window, int32_t sinks, void* out, int32_t ldo, void* workspace, size_t workspace_bytes,
                       int32_t dtype, void* stream, const char* fn) {
    rag::PlanView v;
    rag_status st;
    if ((st = check_window(plan, v, keys.max_len, kv_heads, window, sinks, dtype, fn))) return st;
    if (head_dim != RAG_HEAD_DIM) return fail(RAG_ERR_SHAPE, "%s: head_dim %d unsupported (only %d)", fn, head_dim, RAG_HEAD_DIM);
    if (!std::isfinite(scale)) return fail(RAG_ERR_ARG, "%s: scale is not finite", fn);
    const int64_t T = plan->total_tokens, wq = (int64_t)plan->heads * head_dim, wk = (int64_t)kv_heads * head_dim;
    if (T == 0) return RAG_OK;  // nothing is read or written
    if ((st = check_rows(q, ldq, wq, dtype, "q", fn)) || (st = check_rows(out, ldo, wq, dtype, "out", fn))) return st;
    if (keys.rows > 0 &&
        ((st = check_rows(k, ldk, wk, dtype, "k", fn)) || (st = check_rows(vv, ldv, wk, dtype, "v", fn)))) return st;
    if (ldq >= kWindowMaxLd || ldk >= kWindowMaxLd || ldv >= kWindowMaxLd || ldo >= kWindowMaxLd)
        return fail(RAG_ERR_SHAPE, "%s: a leading dimension is not below %d", fn, kWindowMaxLd);
    const int splits = rag::window_splits(T, plan->batch, plan->heads, kv_heads, plan->max_len, keys.max_len, window, sinks);
    const size_t need = rag::window_workspace(T, plan->heads, splits);
    if (need > 0) {
        if (workspace_bytes < need)
            return fail(RAG_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, workspace_bytes, need);
        if (!workspace || !aligned(workspace, 16)) return fail(RAG_ERR_ARG, "%s: workspace NULL or misaligned", fn);
    }
    const Span so{out, span_bytes(T, ldo, wq, dtype), ldo}, sw{need ? workspace : nullptr, need, -2};
    const Span in[5] = {{q, span_bytes(T, ldq, wq, dtype), -1}, {k, span_bytes(keys.rows, ldk, wk, dtype), -1},
                        {vv, span_bytes(keys.rows, ldv, wk, dtype), -1},
                        {keys.first, keys.first ? 8 * (size_t)plan->batch : 0, -1}, {keys.len, keys.len ? 4 * (size_t)plan->batch : 0, -1}};
    for (const Span& i : in)
        if (clash(so, i) || clash(sw, i)) return fail(RAG_ERR_ARG, "%s: out or the workspace overlaps an input", fn);
    if (clash(so, sw)) return fail(RAG_ERR_ARG, "%s: out overlaps the workspace", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return finish(rag::launch_attention_window(v, dtype, q, ldq, k, ldk, vv, ldv, keys, kv_heads, scale, window, sinks, out,
                                               ldo, splits, need ? workspace : nullptr, s),
                  s, plan->status, fn);
}

}  // namespace

rag_status ragged_attention_window_workspace(const rag_plan* plan, int32_t max_kv_len, int32_t kv_heads, int32_t window,
                                             int32_t sinks, int32_t dtype, size_t* bytes) {
    const char* fn = "ragged_attention_window_workspace";
    rag::PlanView v;
    if (!bytes) return fail(RAG_ERR_ARG, "%s: output pointer is NULL", fn);
    const rag_status st = check_window(plan, v, max_kv_len, kv_heads, window, sinks, dtype, fn);
    if (st) return st;
    *bytes = rag::window_workspace(plan->total_tokens, plan->heads,
                                   rag::window_splits(plan->total_tokens, plan->batch, plan->heads, kv_heads, plan->max_len,
                                                      max_kv_len, window, sinks));
    return RAG_OK;
}

rag_status ragged_attention_window(const rag_plan* plan, const void* q, int32_t ldq, const void* k, int32_t ldk,
                                   const void* v, int32_t ldv, int32_t kv_heads, int32_t head_dim, float scale,
                                   int32_t window, int32_t sinks, void* out, int32_t ldo, void* workspace,
                                   size_t workspace_bytes, int32_t dtype, void* stream) {
    const rag::WindowKeys keys{nullptr, nullptr, plan ? plan->total_tokens : 0, plan ? plan->max_len : 0};
    return window_impl(plan, q, ldq, k, ldk, v, ldv, keys, kv_heads, head_dim, scale, window, sinks, out, ldo, workspace,
                       workspace_bytes, dtype, stream, "ragged_attention_window");
}

rag_status ragged_attention_window_cached(const rag_plan* plan, const void* q, int32_t ldq, const void* k, int32_t ldk,
                                          const void* v, int32_t ldv, int64_t kv_rows, const int64_t* kv_first,
                                          const int32_t* kv_len, int32_t max_kv_len, int32_t kv_heads, int32_t head_dim,
                                          float scale, int32_t window, int32_t sinks, void* out, int32_t ldo,
                                          void* workspace, size_t workspace_bytes, int32_t dtype, void* stream) {
    const char* fn = "ragged_attention_window_cached";
    if (kv_rows < 0 || kv_rows > ((int64_t)1 << 40)) return fail(RAG_ERR_ARG, "%s: kv_rows %lld out of range", fn, (long long)kv_rows);
    if (!kv_first || !kv_len || !aligned(kv_first, 8) || !aligned(kv_len, 4))
        return fail(RAG_ERR_ARG, "%s: kv_first or kv_len NULL or misaligned", fn);
    const rag::WindowKeys keys{kv_first, kv_len, kv_rows, max_kv_len};
    return window_impl(plan, q, ldq, k, ldk, v, ldv, keys, kv_heads, head_dim, scale, window, sinks, out, ldo, workspace,
                       workspace_bytes, dtype, stream, fn);
}

}  // extern "C"
