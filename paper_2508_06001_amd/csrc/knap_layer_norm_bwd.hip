// Layer norm, backward (knap_layer_norm.h), with g = dy w and xh = (x - mean) rstd:
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy.
// Bound by HBM: x and dy are read once, dx is written once.  A workgroup stays for its share of the rows and holds its dw and db in
// registers; they go to the workspace as one row of sums a workgroup, which a second kernel adds up in a fixed order: no atomics,
// the same bits every time.
// Measured, with the second kernel behind the +: 31464 rows of 1536, bf16, 47 + 5 us (6.1 TB/s); 103008 of 128 17 + 4 us (4.7); 8191 of 4099, 32 bits,
// dy of 16, 60 + 5 us (5.6); 37 of 768 5 + 2.5 us.
#include "knap_layer_norm.h"

#include <algorithm>

namespace knap {

template <class C, class TX, class TY>
__global__ __launch_bounds__(C::THREADS, 2) void layer_norm_bwd_kernel(NormArgs a) {
  __shared__ float s_sum[2][2 * C::ROWS * 8];
  __shared__ float s_cols[C::GROUPS > 1 ? C::THREADS * C::COLS : 1];
  const int g = threadIdx.x % C::LANES, group = threadIdx.x / C::LANES;
  const int width = a.width;
  const float n = (float)width;
  float w[C::COLS], dw[C::COLS], db[C::COLS];
  load_weight<C>(a.weight, a.w_bf16, 1.f, g, width, w);
#pragma unroll
  for (int i = 0; i < C::COLS; ++i) dw[i] = db[i] = 0.f;
  const TX* x_base = static_cast<const TX*>(a.x);
  const TY* dy_base = static_cast<const TY*>(a.dy);
  TX* dx_base = static_cast<TX*>(a.dx);
  const int64_t step = (int64_t)gridDim.x * C::PASS;
  RowRaw<C, TX> next_x[C::ROWS];
  RowRaw<C, TY> next_dy[C::ROWS];
  float next_mean[C::ROWS], next_rstd[C::ROWS];
  auto load = [&](int64_t r0) {
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      const int64_t first = r0 + k * C::GROUPS, row = first + group;
      load_row<C, TX>(RowPlace<C, TX>(x_base, a.x_stride, first, group, a.rows, width), g, next_x[k]);
      load_row<C, TY>(RowPlace<C, TY>(dy_base, a.y_stride, first, group, a.rows, width), g, next_dy[k]);
      next_mean[k] = row < a.rows ? a.mean[row] : 0.f;
      next_rstd[k] = row < a.rows ? a.rstd[row] : 0.f;
    }
  };
  load((int64_t)blockIdx.x * C::PASS);
  int turn = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * C::PASS; r0 < a.rows; r0 += step, turn ^= 1) {
    RowRaw<C, TX> x[C::ROWS];
    RowRaw<C, TY> dy[C::ROWS];
    float sums[2 * C::ROWS], rstd[C::ROWS], shift[C::ROWS];
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      x[k] = next_x[k];
      dy[k] = next_dy[k];
      rstd[k] = next_rstd[k];
      shift[k] = next_mean[k];
    }
    load(r0 + step);
    // columns behind the row's end have dy = 0 and add nothing
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) {
        const float xh = (x[k].get(i) - shift[k]) * rstd[k], y = dy[k].get(i), gi = y * w[i];
        dw[i] = __builtin_fmaf(y, xh, dw[i]);
        db[i] += y;
        s1 += gi;
        s2 = __builtin_fmaf(gi, xh, s2);
      }
      sums[2 * k] = s1;
      sums[2 * k + 1] = s2;
    }
    row_sums<C>(sums, s_sum[turn]);
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      const float m1 = sums[2 * k] / n, m2 = sums[2 * k + 1] / n;
      float dx[C::COLS];
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) {
        const float xh = (x[k].get(i) - shift[k]) * rstd[k];
        dx[i] = rstd[k] * (__builtin_fmaf(dy[k].get(i), w[i], -m1) - xh * m2);
      }
      store_row<C, TX>(RowPlace<C, TX>(dx_base, a.dx_stride, r0 + k * C::GROUPS, group, a.rows, width), g, dx);
    }
  }
  if (!a.partial) return;
  float* mine = a.partial + (size_t)blockIdx.x * 2 * width;
  if constexpr (C::GROUPS == 1) {
#pragma unroll
    for (int i = 0; i < C::COLS; ++i)
      if (norm_has<C>(g, i, width)) {
        mine[norm_col<C>(g, i)] = dw[i];
        mine[width + norm_col<C>(g, i)] = db[i];
      }
  } else {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < C::COLS; ++i)
        if (norm_has<C>(g, i, width)) s_cols[group * width + norm_col<C>(g, i)] = half == 0 ? dw[i] : db[i];
      __syncthreads();
      for (int c = threadIdx.x; c < width; c += C::THREADS) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < C::GROUPS; ++k) sum += s_cols[k * width + c];
        mine[half * width + c] = sum;
      }
    }
  }
}

// sums[c] = sum over `n` rows of partial[.][c], for 2 width columns: COLS columns of a workgroup, its 1024 threads' rows joined in LDS
template <int COLS>
__global__ __launch_bounds__(1024) void layer_norm_sum_kernel(const float* __restrict__ partial, int n, int width, float* __restrict__ dw,
                                                              float* __restrict__ db) {
  constexpr int SLICES = 1024 / COLS;
  __shared__ float s_part[SLICES][COLS];
  const int c = threadIdx.x % COLS, slice = threadIdx.x / COLS;
  const int col = (int)blockIdx.x * COLS + c;
  float sum = 0.f;
  if (col < 2 * width) {
#pragma unroll 8
    for (int r = slice; r < n; r += SLICES) sum += partial[(size_t)r * 2 * width + col];
  }
  s_part[slice][c] = sum;
  __syncthreads();
  if (slice == 0 && col < 2 * width) {
    sum = 0.f;
    for (int k = 0; k < SLICES; ++k) sum += s_part[k][c];
    if (col < width) { if (dw) dw[col] = sum; }
    else if (db) db[col - width] = sum;
  }
}

template <class TX, class TY, bool WIDE>
static hipError_t launch_bwd_t(const NormArgs& a, float* dw, float* db, int cus, hipStream_t stream) {
  return norm_form<WIDE>(a.width, [&](auto cfg) {
    using C = decltype(cfg);
    const int64_t passes = (a.rows + C::PASS - 1) / C::PASS;
    // two workgroups a CU, which is what the registers of the wider forms allow: more of them only leave more sums to add up (8191 rows of
    // 4099 in 32 bits, four -> two, us: 65.0 -> 60.0 and 9.4 -> 5.6 for the sums; 103008 of 128 19.4 -> 18.6; 31464 of 1536 the same, 6.4 -> 5.4)
    const int most = (int)std::min<int64_t>(passes, std::min(2 * cus, kNormMaxGroups));
    const int64_t each = (passes + most - 1) / most;          // as many for every workgroup, but for the last
    const int groups = (int)((passes + each - 1) / each);
    hipLaunchKernelGGL((layer_norm_bwd_kernel<C, TX, TY>), dim3(groups), dim3(C::THREADS), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.partial) return e;
    if (a.width <= 2048)
      hipLaunchKernelGGL(layer_norm_sum_kernel<16>, dim3((2 * a.width + 15) / 16), dim3(1024), 0, stream, a.partial, groups, a.width, dw, db);
    else
      hipLaunchKernelGGL(layer_norm_sum_kernel<64>, dim3((2 * a.width + 63) / 64), dim3(1024), 0, stream, a.partial, groups, a.width, dw, db);
    return hipGetLastError();
  });
}

// gradients of no rows
hipError_t launch_layer_norm_zero(float* dw, float* db, int width, hipStream_t stream) {
  hipLaunchKernelGGL(layer_norm_sum_kernel<64>, dim3((2 * width + 63) / 64), dim3(1024), 0, stream, nullptr, 0, width, dw, db);
  return hipGetLastError();
}

hipError_t launch_layer_norm_bwd(const NormArgs& a, float* dw, float* db, bool x_bf16, bool y_bf16, bool wide, int cus, hipStream_t stream) {
  if (x_bf16) return wide ? launch_bwd_t<__bf16, __bf16, true>(a, dw, db, cus, stream) : launch_bwd_t<__bf16, __bf16, false>(a, dw, db, cus, stream);
  if (y_bf16) return wide ? launch_bwd_t<float, __bf16, true>(a, dw, db, cus, stream) : launch_bwd_t<float, __bf16, false>(a, dw, db, cus, stream);
  return wide ? launch_bwd_t<float, float, true>(a, dw, db, cus, stream) : launch_bwd_t<float, float, false>(a, dw, db, cus, stream);
}

}  // namespace knap
