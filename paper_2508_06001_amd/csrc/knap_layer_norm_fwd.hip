// Layer norm, forward (knap_layer_norm.h): y = (x - mean) rstd w + b, with mean and rstd of every row where a backward follows.
// Bound by HBM: a row is read once and written once.  Workgroups stay for several rows, so that weights and biases are read once each.
// Measured: 31464 rows of 1536, bf16, 34 us (5.7 TB/s); 103008 of 128 11 us (4.9); 8191 of 4099, 32 bits in, 16 out, 42 us (4.8); 37 of 768 3.4 us.
#include "knap_layer_norm.h"

#include <algorithm>

namespace knap {

template <class C, class TX, class TY>
__global__ __launch_bounds__(C::THREADS, 2) void layer_norm_fwd_kernel(NormArgs a) {
  __shared__ float s_sum[2][C::ROWS * 8];
  const int g = threadIdx.x % C::LANES, group = threadIdx.x / C::LANES;
  const int width = a.width;
  const float n = (float)width;      // divided by, not multiplied with 1 / n: the mean of equal values is theirs, whatever their number
  float w[C::COLS], b[C::COLS];
  load_weight<C>(a.weight, a.w_bf16, 1.f, g, width, w);
  load_weight<C>(a.bias, a.w_bf16, 0.f, g, width, b);
  const TX* x_base = static_cast<const TX*>(a.x);
  TY* y_base = static_cast<TY*>(a.y);
  const int64_t step = (int64_t)gridDim.x * C::PASS;
  RowRaw<C, TX> next[C::ROWS];
  auto load = [&](int64_t r0) {
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) load_row<C, TX>(RowPlace<C, TX>(x_base, a.x_stride, r0 + k * C::GROUPS, group, a.rows, width), g, next[k]);
  };
  load((int64_t)blockIdx.x * C::PASS);
  for (int64_t r0 = (int64_t)blockIdx.x * C::PASS; r0 < a.rows; r0 += step) {
    RowRaw<C, TX> x[C::ROWS];
    float sum[C::ROWS], mean[C::ROWS];
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) x[k] = next[k];
    load(r0 + step);
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      sum[k] = 0.f;
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) sum[k] += x[k].get(i);
    }
    row_sums<C>(sum, s_sum[0]);
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      mean[k] = sum[k] / n;
      sum[k] = 0.f;
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) {
        const float d = norm_has<C>(g, i, width) ? x[k].get(i) - mean[k] : 0.f;
        sum[k] = __builtin_fmaf(d, d, sum[k]);
      }
    }
    row_sums<C>(sum, s_sum[1]);
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      const float rstd = 1.0f / sqrtf(sum[k] / n + a.eps);
      float y[C::COLS];
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) y[i] = __builtin_fmaf((x[k].get(i) - mean[k]) * rstd, w[i], b[i]);
      store_row<C, TY>(RowPlace<C, TY>(y_base, a.y_stride, r0 + k * C::GROUPS, group, a.rows, width), g, y);
      const int64_t row = r0 + k * C::GROUPS + group;
      if (g == 0 && row < a.rows) {
        if (a.mean) a.mean[row] = mean[k];
        if (a.rstd) a.rstd[row] = rstd;
      }
    }
  }
}

template <class TX, class TY, bool WIDE>
static hipError_t launch_fwd_t(const NormArgs& a, int cus, hipStream_t stream) {
  return norm_form<WIDE>(a.width, [&](auto cfg) {
    using C = decltype(cfg);
    const int64_t passes = (a.rows + C::PASS - 1) / C::PASS;
    hipLaunchKernelGGL((layer_norm_fwd_kernel<C, TX, TY>), dim3((unsigned)std::min<int64_t>(passes, 8 * cus)), dim3(C::THREADS), 0, stream, a);
    return hipGetLastError();
  });
}

hipError_t launch_layer_norm_fwd(const NormArgs& a, bool x_bf16, bool y_bf16, bool wide, int cus, hipStream_t stream) {
  if (x_bf16) return wide ? launch_fwd_t<__bf16, __bf16, true>(a, cus, stream) : launch_fwd_t<__bf16, __bf16, false>(a, cus, stream);
  if (y_bf16) return wide ? launch_fwd_t<float, __bf16, true>(a, cus, stream) : launch_fwd_t<float, __bf16, false>(a, cus, stream);
  return wide ? launch_fwd_t<float, float, true>(a, cus, stream) : launch_fwd_t<float, float, false>(a, cus, stream);
}

}  // namespace knap
