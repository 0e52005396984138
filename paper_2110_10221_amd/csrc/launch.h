// Host-side launchers of the HIP kernels.  Each .hip file defines its kernels
// and the launchers below; api.cpp validates arguments and calls them.  Every
// launcher enqueues work on `stream` and returns the launch error (if any).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ragged.h"

namespace rag {

struct PlanView {
    int32_t batch, total_tokens, max_len, heads;
    int64_t qkt_cap, av_cap;
    const int32_t* lengths;
    int32_t* tok_off;
    int64_t* att_off;
    int32_t* order;
    int32_t* tok_seq;
    int32_t* qkt_item_off;
    int32_t* av_item_off;
    int32_t* qkt_items;
    int32_t* av_items;
    int32_t* status;
};

// Number of compute units of the current device (cached per device).
int device_cu_count();

// Record a formatted message as the thread's last error and return `status`.
rag_status report(rag_status status, const char* fmt, ...);

hipError_t launch_offsets(const PlanView& p, hipStream_t s);

// Attention operators; dtype 0 = fp32, 1 = bf16.  Persistent grids sized from the
// host-side capacities; item counts are read on the device.
// `causal` selects masked attention (position i sees keys j <= i).
hipError_t launch_qkt(const PlanView& p, int dtype, const void* q, int ldq, const void* k, int ldk,
                      float scale, void* scores, int64_t score_cap, bool causal, hipStream_t s);
hipError_t launch_softmax(const PlanView& p, int dtype, const void* scores, void* probs,
                          int64_t score_cap, bool causal, hipStream_t s);
hipError_t launch_attn_v(const PlanView& p, int dtype, const void* probs, int64_t score_cap,
                         const void* v, int ldv, void* out, int ldo, bool causal, hipStream_t s);
hipError_t launch_fused_attention(const PlanView& p, int dtype, const void* q, int ldq, const void* k,
                                  int ldk, const void* v, int ldv, float scale, void* out, int ldo,
                                  bool causal, hipStream_t s);

// With `plan`, the launch also builds that batch's plan (as launch_offsets does):
// bf16 projections of batches up to 256 sequences carry the prelude's
// workgroups behind their tiles, other cases launch the prelude first.
hipError_t launch_linear(int dtype, const void* x, int ldx, const void* w, const void* bias,
                         const void* residual, int ldr, int act, void* y, int ldy, int T, int K, int N,
                         hipStream_t s, const PlanView* plan = nullptr);

// Variable-sized batched GEMM.  VgemmView mirrors rag_vgemm_plan.
struct VgemmView {
    int32_t batch;
    int64_t tile_cap;
    const int32_t* dims;
    int64_t* a_off;
    int64_t* b_off;
    int64_t* c_off;
    int32_t* order;
    int64_t* tile_off;
    int32_t* tile_items;
    int32_t* status;
};

hipError_t launch_vgemm_offsets(const VgemmView& p, hipStream_t s);
hipError_t launch_vgemm(const VgemmView& p, int dtype, const void* a, int64_t a_cap, const void* b, int64_t b_cap,
                        void* c, int64_t c_cap, hipStream_t s);

// C = tril(L) B: L [n, n] (ldl), B and C [n, m] (ldb, ldc).
hipError_t launch_trmm(int dtype, const void* l, int ldl, const void* b, int ldb, void* c, int ldc, int n, int m,
                       hipStream_t s);

hipError_t launch_layernorm(int dtype, const void* x, int ldx, const void* gamma, const void* beta,
                            float eps, void* y, int ldy, int T, int d, hipStream_t s);

// RMS norm with the residual's addition (residual, sum, y and q may be NULL), and 8-bit rows.
hipError_t launch_rmsnorm(int dtype, const void* x, int ldx, const void* residual, int ldr, const void* gamma, float eps,
                          void* sum, int lds, void* y, int ldy, int8_t* q, int ldq, float* q_scale, int T, int d,
                          hipStream_t s);
hipError_t launch_quantize_i8(int dtype, const void* x, int ldx, int8_t* q, int ldq, float* scale, int T, int d,
                              hipStream_t s);

// Rotary positions of the plan's tokens; inv_freq (fp64) and pos_start are device memory.
hipError_t launch_rotary(const PlanView& p, int dtype, const void* x, int ldx, void* y, int ldy, int heads, int head_dim,
                         int rot_dim, bool half, bool inverse, const double* inv_freq, float amplitude,
                         const int32_t* pos_start, hipStream_t s);

// y = act(x_scale w_scale x w^T + bias) + residual on 8-bit rows; dtype is that of bias, residual and y.
// linear_form_i8: the form of tiles that is modelled fastest for its sizes; linear_kernel_i8: the kernel that runs.
enum { kI8Few, kI8Tiles32x32, kI8Tiles32x64Deep, kI8Tiles32x64, kI8Tiles64x64, kI8Tiles64x128, kI8Tiles128x128, kI8Tiles256x256 };
int linear_form_i8(int64_t T, int64_t K, int64_t N, int act, bool bf16, int64_t cus);
int linear_kernel_i8(int64_t T, int64_t K, int64_t N, int act, bool bf16, int64_t cus);
hipError_t launch_linear_i8(int dtype, const int8_t* x, int ldx, const float* x_scale, const int8_t* w,
                            const float* w_scale, const void* bias, const void* residual, int ldr, int act, void* y,
                            int ldy, int T, int K, int N, hipStream_t s);

// Sliding-window attention.  `first` and `len` NULL: each sequence's keys are its own tokens.
struct WindowKeys {
    const int64_t* first;
    const int32_t* len;
    int64_t rows;
    int32_t max_len;
};
int window_splits(int64_t T, int64_t batch, int64_t heads, int64_t kv_heads, int64_t max_len, int64_t max_kv, int64_t window,
                  int64_t sinks);
size_t window_workspace(int64_t T, int64_t heads, int64_t splits);
hipError_t launch_attention_window(const PlanView& p, int dtype, const void* q, int ldq, const void* k, int ldk,
                                   const void* v, int ldv, const WindowKeys& keys, int kv_heads, float scale, int window,
                                   int sinks, void* out, int ldo, int splits, void* workspace, hipStream_t s);

}  // namespace rag
