// Layer norm of rows, forward and backward: what both directions share.
//   xh = (x - mean) rstd, y = xh w + b
// A row is held by LANES threads in registers (UNITS times 8 columns each), so that it is read once, its mean and then its squared
// distances from it are summed in 32 bits, and nothing is read again.  Up to 2048 columns that is part of a wave or a whole one; wider
// rows take the workgroup, whose waves join their sums in LDS.  ROWS rows are in work at a time, for as many bytes in flight whatever
// the width.  WIDE: 16-byte accesses (a width of whole units of 8 columns, every row on 16 bytes); else one column at a time.
#pragma once

#include "knap_device.h"
#include "knap_kernels.h"

namespace knap {

template <int LANES_, int UNITS_, int ROWS_, bool WIDE_>
struct NormCfg {
  static constexpr int LANES = LANES_, UNITS = UNITS_, ROWS = ROWS_;
  static constexpr bool WIDE = WIDE_;
  static constexpr int THREADS = LANES > 256 ? LANES : 256;
  static constexpr int GROUPS = THREADS / LANES;          // rows side by side
  static constexpr int COLS = 8 * UNITS;                  // of a thread
  static constexpr int PASS = GROUPS * ROWS;              // rows of a workgroup at a time
};

// column of a thread's element i (unit i / 8 of 8 consecutive ones, or every LANES-th)
template <class C>
__device__ __forceinline__ int norm_col(int g, int i) { return C::WIDE ? (g + C::LANES * (i >> 3)) * 8 + (i & 7) : g + C::LANES * i; }

// whether it is one of the row
template <class C>
__device__ __forceinline__ bool norm_has(int g, int i, int width) { return C::WIDE ? (g + C::LANES * (i >> 3)) * 8 < width : g + C::LANES * i < width; }

__device__ __forceinline__ void load8(const __bf16* p, float (&v)[8]) {
  const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __builtin_bit_cast(float, x[e] << 16);
    v[2 * e + 1] = __builtin_bit_cast(float, x[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const f32x4 x = *reinterpret_cast<const f32x4*>(p), y = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[e] = x[e]; v[4 + e] = y[e]; }
}
__device__ __forceinline__ void store8(__bf16* p, const float* v) {
  *reinterpret_cast<bf16x8*>(p) = pack8(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(float* p, const float* v) {
  const f32x4 x = {v[0], v[1], v[2], v[3]}, y = {v[4], v[5], v[6], v[7]};
  *reinterpret_cast<f32x4*>(p) = x;
  *reinterpret_cast<f32x4*>(p + 4) = y;
}

// a row's columns of this thread; zeros where it has none
template <class C, class T>
__device__ __forceinline__ void load_row(const T* row, bool there, int g, int width, float (&v)[C::COLS]) {
#pragma unroll
  for (int u = 0; u < C::UNITS; ++u) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if constexpr (C::WIDE) {
      if (there && norm_has<C>(g, 8 * u, width)) load8(row + norm_col<C>(g, 8 * u), x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (there && norm_has<C>(g, 8 * u + e, width)) x[e] = (float)row[norm_col<C>(g, 8 * u + e)];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[8 * u + e] = x[e];
  }
}

template <class C, class T>
__device__ __forceinline__ void store_row(T* row, bool there, int g, int width, const float (&v)[C::COLS]) {
  if (!there) return;
#pragma unroll
  for (int u = 0; u < C::UNITS; ++u) {
    if constexpr (C::WIDE) {
      if (norm_has<C>(g, 8 * u, width)) store8(row + norm_col<C>(g, 8 * u), v + 8 * u);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (norm_has<C>(g, 8 * u + e, width)) row[norm_col<C>(g, 8 * u + e)] = (T)v[8 * u + e];
    }
  }
}

// weight or bias columns of this thread, `none` where there is no such vector
template <class C>
__device__ __forceinline__ void load_weight(const void* w, bool w_bf16, float none, int g, int width, float (&v)[C::COLS]) {
#pragma unroll
  for (int i = 0; i < C::COLS; ++i) v[i] = none;
  if (!w) return;
  if constexpr (C::WIDE) {
    if ((reinterpret_cast<uintptr_t>(w) & 15) == 0) {
#pragma unroll
      for (int u = 0; u < C::UNITS; ++u)
        if (norm_has<C>(g, 8 * u, width)) {
          float x[8];
          if (w_bf16) load8(static_cast<const __bf16*>(w) + norm_col<C>(g, 8 * u), x);
          else load8(static_cast<const float*>(w) + norm_col<C>(g, 8 * u), x);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[8 * u + e] = x[e];
        }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < C::COLS; ++i)
    if (norm_has<C>(g, i, width)) {
      const int c = norm_col<C>(g, i);
      v[i] = w_bf16 ? (float)static_cast<const __bf16*>(w)[c] : static_cast<const float*>(w)[c];
    }
}

// N sums over the threads of a row, in every one of them.  s_sum: waves x N floats, another place than that of the call before.
template <class C, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float* s_sum) {
#pragma unroll
  for (int o = 1; o < (C::LANES < 64 ? C::LANES : 64); o <<= 1)
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] += __shfl_xor(x[n], o, 64);
  if constexpr (C::LANES > 64) {
    constexpr int WAVES = C::THREADS / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) s_sum[N * wave + n] = x[n];
    }
    lds_barrier();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      x[n] = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) x[n] += s_sum[N * w + n];
    }
  }
}

// Which form a width takes: the fewest threads of a row whose registers hold it.  f(cfg) is called with the form.
template <bool WIDE, class F>
hipError_t norm_form(int width, F f) {
  if constexpr (WIDE) {
    if (width <= 128) return f(NormCfg<16, 1, 4, WIDE>{});
    if (width <= 256) return f(NormCfg<32, 1, 4, WIDE>{});
  }
  if (width <= 512) return f(NormCfg<64, 1, 4, WIDE>{});
  if (width <= 1024) return f(NormCfg<64, 2, 2, WIDE>{});
  if (width <= 2048) return f(NormCfg<64, 4, 1, WIDE>{});
  if (width <= 4096) return f(NormCfg<256, 2, 2, WIDE>{});
  if (width <= 8192) return f(NormCfg<256, 4, 1, WIDE>{});
  return f(NormCfg<512, 4, 1, WIDE>{});
}

}  // namespace knap
