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

// resident workgroups per compute unit of the persistent kernels
int fwd_workgroups_per_cu(int d);
int bwd_dq_workgroups_per_cu(int d);

}  // namespace knap
