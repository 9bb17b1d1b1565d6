// Internal launch interface between the C-ABI layer and the kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "knap_dispatch.h"
#include "knapattn.h"

namespace knap {

// the forward without the mask (knap_attn_fwd_full.hip) and the causal one (knap_attn_fwd.hip)
hipError_t launch_fwd_full(const void* q, const void* k, const void* v, const int32_t* cu, int n_seq, int H, int d, float scale,
                           void* out, float* lse, unsigned* counters, int grid, hipStream_t stream);
hipError_t launch_fwd_causal(const void* q, const void* k, const void* v, const int32_t* cu, int n_seq, int H, int d, float scale,
                             void* out, float* lse, unsigned* counters, int grid, hipStream_t stream);

// Device address (on the current device) of the forward's work-queue counters: kQueueSets sets of 8, at zero
// whenever no kernel uses them; nullptr on failure.
unsigned* queue_base();
hipError_t clear_queue_sets(unsigned* first, unsigned sets, hipStream_t stream);

struct BwdArgs {
  const void *q, *k, *v, *out, *dout;
  const float* lse;
  const int32_t* cu;
  int n_seq, H;
  float scale;
  void *dq, *dk, *dv;
  float *delta, *lse2;      // (H, T) each, -delta and the base-2 LSE, handed from the dQ kernel to the dK/dV kernel
  unsigned* counters;       // 8 for the dQ kernel, 8 for the dK/dV kernel; the launches clear them, they may hold anything
};
// `dkdv_pairs`: wave pairs (2 or 4) per workgroup of the dK/dV kernel
hipError_t launch_bwd(const BwdArgs& a, int d, bool causal, int dkdv_pairs, int cus, int dq_wg_per_cu, hipStream_t stream,
                      hipEvent_t ev_start, hipEvent_t ev_stop);
// both kinds of items in one launch, T tokens, behind the kernel that forms delta: tiles of 128 rows (knap_attn_joint.h) or, `small`, of 64
// (knap_attn_bwd_small.hip)
constexpr int kSmallPays = 8;      // behind the counters of the launch's queues: whether items of 64 rows pay, where that is decided on the device
hipError_t launch_joint(const BwdArgs& a, int d, bool causal, bool small, int T, int cus, hipStream_t stream, hipEvent_t ev_start,
                        hipEvent_t ev_stop);
hipError_t launch_small(const BwdArgs& a, int d, bool causal, bool sure, int cus, hipStream_t stream);
hipError_t launch_joint_causal(const BwdArgs& a, int d, int cus, hipStream_t stream);
hipError_t launch_dq_causal(const BwdArgs& a, int d, int cus, int wg_per_cu, hipStream_t stream);
hipError_t launch_dkdv_causal(const BwdArgs& a, int d, int pairs, int cus, hipStream_t stream);

// Ulysses layout switch, local data movement; rows of U 16-byte units.
hipError_t launch_ulysses_heads(const void* src, void* dst, uint32_t T, uint32_t U, uint32_t g, bool pack,
                                hipStream_t stream);
hipError_t launch_ulysses_rows(const void* src, void* dst, const int32_t* row_map, uint32_t T, uint32_t U,
                               bool gather, hipStream_t stream);
hipError_t launch_ulysses_plan(const int32_t* cu, int n_seq, int g, int T, int32_t* row_map, hipStream_t stream);

// Differential attention
struct DiffFwdArgs {
  const __bf16 *q, *k, *v;
  const int32_t* cu;
  int n_seq, H;
  float scale;
  const float* lambda;      // (H)
  __bf16 *out, *out2;       // out2 (the second map's output) or nullptr
  float* lse;               // (2, H, T)
  unsigned* counters;
};
struct DiffBwdArgs {
  const __bf16 *q, *k, *v, *out, *out2, *dout;
  const int32_t* cu;
  int n_seq, H;
  float scale;
  const float *lambda, *lse;
  __bf16 *dq, *dk, *dv;
  float* dlambda;
  float *nd1, *diff, *lse_a, *lse_b, *d2;      // (H, T) each: -D_1, D_1 - D_2, the log-sums in base 2 less 15, D_2 in 32 bits
  unsigned* counters;                          // 8 for the dK/dV kernel, which the dQ kernel clears
  unsigned* dq_counters;                       // a set of the forward's, at zero
};
hipError_t launch_diff_fwd(const DiffFwdArgs& a, int d, bool causal, int cus, hipStream_t stream);
hipError_t launch_diff_bwd(const DiffBwdArgs& a, int d, bool causal, int tokens, int cus, hipStream_t stream);

// Rotary positions: everything but the launch geometry comes from the caller
struct RopeArgs {
  const __bf16 *q, *k;
  __bf16 *q_out, *k_out;
  int64_t q_token, q_head, k_token, k_head, qo_token, qo_head, ko_token, ko_head;      // strides in elements
  int T, H, Hk, d, rot;
  const int32_t* positions;      // (T, n_axes), or nullptr: by cu
  int n_axes, axis_end[KNAP_ROPE_MAX_AXES];      // the first pair that is not of the axis
  const int32_t* cu;
  int n_seq;
  const double* freq;
  float factor, sign;      // sign: of the sine
  bool copies;             // columns from rot on go to another tensor
  int tokens_per_group, first_group;    // set by the launch
};
hipError_t launch_rope(RopeArgs a, bool half, bool aligned, int cus, hipStream_t stream);

// Layer norm
struct NormArgs {
  const void *x, *weight, *bias, *dy;
  void *y, *dx;
  float *mean, *rstd, *partial;      // partial: (workgroups, 2, width), the sums of dy xh and of dy
  int64_t x_stride, y_stride, dx_stride, rows;      // y_stride: of y or dy
  int width;
  float eps;
  bool w_bf16;
};
constexpr int kNormMaxGroups = 1024;      // workgroups of a backward
hipError_t launch_layer_norm_fwd(const NormArgs& a, bool x_bf16, bool y_bf16, bool wide, int cus, hipStream_t stream);
hipError_t launch_layer_norm_bwd(const NormArgs& a, float* dw, float* db, bool x_bf16, bool y_bf16, bool wide, int cus, hipStream_t stream);
hipError_t launch_layer_norm_zero(float* dw, float* db, int width, hipStream_t stream);

// Residual norm; pointers that are not wanted, and tensors that there are none of, are nullptr
struct ResidualArgs {
  const void *x, *f, *gate, *scale, *shift, *weight, *post_weight, *dx_out, *dy;
  const int32_t* cu;      // or nullptr: one sequence of all rows
  int n_seq;
  void *x_out, *y, *dx, *df;
  float *stats;           // (4, rows): mean and rstd of x', mean and rstd of f
  float *dgate, *dscale, *dshift, *dweight, *dpost_weight;
  float *partial, *totals;      // (workgroups + n_seq, 3, width), (workgroups, 2, width)
  int64_t x_stride, f_stride, x_out_stride, y_stride, dx_out_stride, dy_stride, dx_stride, df_stride;
  int64_t gate_stride, mod_stride, dgate_stride, dmod_stride;
  int64_t rows;
  int width, chunk;       // chunk: rows of a workgroup, set by the launch
  float alpha, eps;
  int norm, post_norm;
  bool w_bf16, mod_bf16;
};
constexpr int kResidualMaxGroups = 768;      // workgroups of a backward
hipError_t launch_residual_norm_fwd(const ResidualArgs& a, bool x_bf16, bool b_bf16, bool wide, int cus, hipStream_t stream);
hipError_t launch_residual_norm_bwd(const ResidualArgs& a, bool x_bf16, bool b_bf16, bool wide, int cus, hipStream_t stream);

// Gradient norm and clipping: a record of the plan stands for up to KNAP_GRAD_CHUNK elements of one tensor
struct GradChunk {
  const void* from;
  void* to;
  int32_t count;
  int32_t bf16;
};
constexpr int kGradGroups = 1024;      // most workgroups of a sum, one double each
static_assert(KNAP_GRAD_WORKSPACE_BYTES == kGradGroups * sizeof(double), "a double a workgroup");
hipError_t launch_grad_squares(const GradChunk* plan, int64_t chunks, double* partial, double* sum, int cus, hipStream_t stream);
hipError_t launch_grad_clip(const GradChunk* plan, int64_t chunks, const double* sum, float max_norm, float eps, float* norm, int cus, hipStream_t stream);

// Matrix products of the gated feed-forward block (knap_gemm.h).  One product of a launch:
struct GemmProblem {
  const __bf16 *a[2], *b[2];      // of the segments of k; a pair of products: b of the first and of the second
  __bf16* c;
  int64_t lda, ldb, ldc;
  int M, N, K;
  int segments;                   // 1 or 2 products of K each, added up
  int tiles_m, tiles_n;
  int step;                       // columns of a tile, of each of a pair
};
struct GemmLaunch {
  GemmProblem p[3];
  int first[3];             // tiles in front of a product's
  int n;                    // products
  int whole, tail, splits;  // tiles that a workgroup forms alone; the others, in `splits` parts of their steps
  float* partial;           // of the parts
  // epilogues: activations' inputs and outputs, (tokens, hidden)
  const __bf16 *gate_in, *up_in;
  __bf16 *gate, *up, *h;
  bool gelu;
  bool keep;                // h, da and db go through the caches
};
struct FfnArgs {
  const __bf16 *x, *w_gate, *w_up, *w_down, *dy;
  int64_t x_stride, y_stride, dy_stride, dx_stride;
  int tokens, width, hidden;
  bool gelu;
  __bf16 *gate, *up, *h, *y;      // gate, up (forward): or nullptr
  __bf16 *dgate, *dup, *dx, *dw_gate, *dw_up, *dw_down;
  float* partial;
};
size_t ffn_partial_bytes(int64_t tokens, int width, int hidden, bool backward);
// Whether a forward takes the form of knap_ffn_few.hip: up to 16 tokens, and up to 32 of smaller weights; it reads the second 16 tokens as often as there
// are workgroups, which tiles do not (us, this form and tiles: 768 x 2048, 32 tokens 14.7 and 21.9; 2048 x 5504, 17 tokens 30 and 34, 24 34 and 34, 32 38 and
// 34; 4096 x 10944, 16 tokens 68.5 and 69.8, 24 80 and 70; 4096 x 16384, 16 tokens 93 and 102, 17 101 and 102).
inline bool ffn_few(int64_t tokens, int64_t width, int64_t hidden) { return tokens <= 16 || (tokens <= 32 && tokens * width * hidden <= 270000000); }
hipError_t launch_ffn_few(const FfnArgs& a, hipStream_t stream);
hipError_t launch_ffn_fwd(const FfnArgs& a, hipStream_t stream);
hipError_t launch_ffn_bwd(const FfnArgs& a, hipStream_t stream);

// for entry points in other files than knap_api.hip: compute units of the current device, 0 where they could not be looked up (as for the
// forward of attention, the first call on a device asks the runtime), and the status of a launch, which is kept for knap_last_hip_error
int device_cus();
int launch_status(hipError_t e);

// resident workgroups per compute unit of the persistent kernels
int fwd_workgroups_per_cu(int d);
int bwd_dq_workgroups_per_cu(int d);

}  // namespace knap
