// Residual norm, forward, over the rows of a packed bag (vectors of the row's sequence: gate, scale, shift):
//   fh = N_post(f),  x' = x + alpha gate (fh wp),  xh = N(x'),  y = xh w (1 + scale) + shift
// with N_post and N each nothing, RMS (x rsqrt(mean x^2 + eps)) or layer norm.  x' is normed before it is rounded to its type.
// Bound by HBM: x and f are read once, x' and y written once.  31464 rows of 1536 in bf16, layer norm, modulated: 387 MB in 73 us (5.3 TB/s); 24576 of 2048,
// x in 32 bits, RMS on both sides: 604 MB in 131 (4.6); 7584 of 1003 in 32 bits, columns singly: 122 MB in 27 (4.5); five rows of 768: 4.8 us.  These are of one
// set of inputs, part of which stays in the last cache; of three in turn, in no cache: 84 us (4.6), 138 (4.4) and 28.
#include "knap_residual_norm.h"

#include <algorithm>

namespace knap {

// mean (layer norm alone) and rstd of ROWS rows that the threads hold
template <class C>
__device__ __forceinline__ void row_stats(const float (&x)[C::ROWS][C::COLS], bool layer, int g, int width, float eps, float (*s_sum)[C::ROWS * C::THREADS / 64],
                                          int& turn, float (&mean)[C::ROWS], float (&rstd)[C::ROWS]) {
  const float n = (float)width;
  float sum[C::ROWS];
  if (layer) {
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      sum[k] = 0.f;
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) sum[k] += x[k][i];
    }
    row_sums<C>(sum, s_sum[turn]);
    turn ^= 1;
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) mean[k] = sum[k] / n;
  } else {
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) mean[k] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < C::ROWS; ++k) {
    sum[k] = 0.f;
#pragma unroll
    for (int i = 0; i < C::COLS; ++i) {
      const float d = norm_has<C>(g, i, width) ? x[k][i] - mean[k] : 0.f;
      sum[k] = __builtin_fmaf(d, d, sum[k]);
    }
  }
  row_sums<C>(sum, s_sum[turn]);
  turn ^= 1;
#pragma unroll
  for (int k = 0; k < C::ROWS; ++k) rstd[k] = 1.0f / sqrtf(sum[k] / n + eps);
}

template <class C, class TX, class TB, bool POST>
__global__ __launch_bounds__(C::THREADS, C::THREADS > 512 ? 4 : 2) void residual_norm_fwd_kernel(ResidualArgs a) {
  __shared__ float s_sum[2][C::ROWS * C::THREADS / 64];
  constexpr bool AHEAD = residual_ahead<C, TX>();
  const int g = threadIdx.x % C::LANES, group = threadIdx.x / C::LANES;
  const int width = a.width;
  const TX* x_base = static_cast<const TX*>(a.x);
  const TB* f_base = static_cast<const TB*>(a.f);
  TX* xo_base = static_cast<TX*>(a.x_out);
  TB* y_base = static_cast<TB*>(a.y);
  RowCursor at;
  at.start(a, (int)min((int64_t)blockIdx.x * a.chunk, a.rows), (int)min((int64_t)(blockIdx.x + 1) * a.chunk, a.rows));
  RowRaw<C, TX> raw_x[C::ROWS];
  RowRaw<C, TB> raw_f[C::ROWS];
  auto load = [&](const RowCursor& c) {
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      const int64_t first = (int64_t)c.row + k * C::GROUPS;
      load_row<C, TX>(RowPlace<C, TX>(x_base, a.x_stride, first, group, c.end, width), g, raw_x[k]);
      if (f_base) load_row<C, TB>(RowPlace<C, TB>(f_base, a.f_stride, first, group, c.end, width), g, raw_f[k]);
    }
  };
  if (AHEAD && at.row < at.limit) load(at);
  int seq = -1, turn = 0;
  float gz[C::COLS], sw[C::COLS], sh[C::COLS];
  while (at.row < at.limit) {
    if (!AHEAD) load(at);
    if (at.seq != seq) {
      seq = at.seq;
      int own = g;      // addresses that are formed here and not outside of the loop, where they would take registers
      asm volatile("" : "+v"(own));
      if (f_base) load_gate<C>(a, seq, own, gz);
      if (y_base) {
        load_scale<C>(a, seq, own, sw);
        const char* shift = a.shift ? static_cast<const char*>(a.shift) + (int64_t)seq * a.mod_stride * (a.mod_bf16 ? 2 : 4) : nullptr;
        load_weight<C>(shift, a.mod_bf16, 0.f, own, width, sh);
      }
    }
    float x[C::ROWS][C::COLS], f[C::ROWS][C::COLS];
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k)
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) {
        x[k][i] = raw_x[k].get(i);
        if (f_base) f[k][i] = raw_f[k].get(i);
      }
    const RowCursor now = at;
    at.step(a, C::PASS);
    if (AHEAD && at.row < at.limit) load(at);
    float mean[C::ROWS], rstd[C::ROWS];
    if (f_base) {
      if constexpr (POST) {
        row_stats<C>(f, a.post_norm == KNAP_NORM_LAYER, g, width, a.eps, s_sum, turn, mean, rstd);
#pragma unroll
        for (int k = 0; k < C::ROWS; ++k) {
          const int64_t row = (int64_t)now.row + k * C::GROUPS + group;
          if (a.stats && g == 0 && row < now.end) {
            a.stats[2 * a.rows + row] = mean[k];
            a.stats[3 * a.rows + row] = rstd[k];
          }
#pragma unroll
          for (int i = 0; i < C::COLS; ++i) f[k][i] = (f[k][i] - mean[k]) * rstd[k];
        }
      }
#pragma unroll
      for (int k = 0; k < C::ROWS; ++k) {
#pragma unroll
        for (int i = 0; i < C::COLS; ++i) x[k][i] = __builtin_fmaf(f[k][i], gz[i], x[k][i]);
        store_row<C, TX>(RowPlace<C, TX>(xo_base, a.x_out_stride, (int64_t)now.row + k * C::GROUPS, group, now.end, width), g, x[k]);
      }
    }
    if (!y_base) continue;
    row_stats<C>(x, a.norm == KNAP_NORM_LAYER, g, width, a.eps, s_sum, turn, mean, rstd);
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      float y[C::COLS];
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) y[i] = __builtin_fmaf((x[k][i] - mean[k]) * rstd[k], sw[i], sh[i]);
      store_row<C, TB>(RowPlace<C, TB>(y_base, a.y_stride, (int64_t)now.row + k * C::GROUPS, group, now.end, width), g, y);
      const int64_t row = (int64_t)now.row + k * C::GROUPS + group;
      if (a.stats && g == 0 && row < now.end) {
        a.stats[row] = mean[k];
        a.stats[a.rows + row] = rstd[k];
      }
    }
  }
}

template <class TX, class TB, bool WIDE>
static hipError_t launch_fwd_t(ResidualArgs a, int cus, hipStream_t stream) {
  return residual_form<WIDE>(a.width, [&](auto cfg) {
    using C = decltype(cfg);
    a.chunk = residual_chunk(a.rows, 4 * cus, C::PASS);
    hipLaunchKernelGGL((a.post_norm == KNAP_NORM_NONE ? residual_norm_fwd_kernel<C, TX, TB, false> : residual_norm_fwd_kernel<C, TX, TB, true>), dim3((unsigned)((a.rows + a.chunk - 1) / a.chunk)), dim3(C::THREADS), 0, stream, a);
    return hipGetLastError();
  });
}

hipError_t launch_residual_norm_fwd(const ResidualArgs& a, bool x_bf16, bool b_bf16, bool wide, int cus, hipStream_t stream) {
  if (x_bf16) return wide ? launch_fwd_t<__bf16, __bf16, true>(a, cus, stream) : launch_fwd_t<__bf16, __bf16, false>(a, cus, stream);
  if (b_bf16) return wide ? launch_fwd_t<float, __bf16, true>(a, cus, stream) : launch_fwd_t<float, __bf16, false>(a, cus, stream);
  return wide ? launch_fwd_t<float, float, true>(a, cus, stream) : launch_fwd_t<float, float, false>(a, cus, stream);
}

}  // namespace knap
