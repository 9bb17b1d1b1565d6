// Layer norm of rows, forward and backward: what both directions share.
//   xh = (x - mean) rstd, y = xh w + b
// A row is held by LANES threads in registers (UNITS times 8 columns each), so that it is read once, its mean and then its squared
// distances from it are summed in 32 bits, and nothing is read again.  Up to 2048 columns that is part of a wave or a whole one; wider
// rows take the workgroup, whose waves join their sums in LDS.  ROWS rows are in work at a time, for as many bytes in flight whatever
// the width.  WIDE: 16-byte accesses (a width of whole units of 8 columns, every row on 16 bytes); else one column at a time.
#pragma once

#include "knap_device.h"
#include "knap_kernels.h"
#include "knap_row_span.h"

#include <type_traits>

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

// A thread's columns of a row as they lie in memory, so that the loads of the next rows can be under way while this one is worked on
// and columns of 16 bits take half a register each.  Columns behind the row's end are zeros: accesses go through a descriptor of the
// row (of the rows of the waves, where several share one), which costs no branches.
template <class C, class T>
struct RowRaw {
  static constexpr bool PACKED = C::WIDE && sizeof(T) == 2;
  static constexpr int WORDS = PACKED ? 4 * C::UNITS : C::COLS;
  uint32_t w[WORDS];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (PACKED) return __builtin_bit_cast(float, (i & 1) ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    else if constexpr (sizeof(T) == 2) return __builtin_bit_cast(float, w[i] << 16);
    else return __builtin_bit_cast(float, w[i]);
  }
};

// rows [row, row + GROUPS) of which the thread's group has the `group`-th; `rows` and `stride` of the tensor
template <class C, class T>
struct RowPlace {
  __amdgpu_buffer_rsrc_t r;
  RowSpan span;
  static constexpr uint32_t SIZE = sizeof(T);
  __device__ __forceinline__ RowPlace(const T* base, int64_t stride, int64_t row0, int group, int64_t rows, int width)
      : span(C::LANES >= 64 ? 0 : group, C::LANES >= 64 ? 1 : min((int64_t)C::GROUPS, rows - row0), stride, width, SIZE) {
    if constexpr (C::LANES >= 64) {
      const int64_t row = row0 + __builtin_amdgcn_readfirstlane(group);
      r = make_rsrc(base + row * stride, row < rows ? (uint32_t)width * SIZE : 0u);
    } else {              // the rows of all groups, at most 2^22 columns apart, or the form is not taken
      r = make_rsrc(base + row0 * stride, RowSpan::bytes(min((int64_t)C::GROUPS, rows - row0), stride, width, SIZE));
    }
  }
  // the byte offset of column c, or one behind everything for columns that the row does not have
  __device__ __forceinline__ int at(int c) const {
    if constexpr (C::LANES >= 64) return c * (int)SIZE;
    else return span.at((uint32_t)c * SIZE);
  }
};

template <class C, class T>
__device__ __forceinline__ void load_row(const RowPlace<C, T>& p, int g, RowRaw<C, T>& v) {
#pragma unroll
  for (int u = 0; u < C::UNITS; ++u) {
    if constexpr (C::WIDE) {
      const int o = p.at(norm_col<C>(g, 8 * u));
#pragma unroll
      for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(p.r, o + 16 * h, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) v.w[(sizeof(T) == 2 ? 4 : 8) * u + 4 * h + e] = x[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int o = p.at(norm_col<C>(g, 8 * u + e));
        v.w[8 * u + e] = sizeof(T) == 2 ? (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(p.r, o, 0, 0) : __builtin_amdgcn_raw_buffer_load_b32(p.r, o, 0, 0);
      }
    }
  }
}

// Stores past the caches, us: 31464 rows of 1536, backward 54.1 -> 47.3; 103008 of 128 12.6 -> 11.3 and 18.6 -> 17.1; 8191 of 4099, 32 bits, 46.0 -> 43.6
// and the same (loads as well: 51.8; 13.1 and 19.1; 44.9 and 70.8).
constexpr int kPast = 2;      // the non-temporal bit of a buffer access
template <class C, class T>
__device__ __forceinline__ void store_row(const RowPlace<C, T>& p, int g, const float (&v)[C::COLS]) {
#pragma unroll
  for (int u = 0; u < C::UNITS; ++u) {
    if constexpr (C::WIDE) {
      const int o = p.at(norm_col<C>(g, 8 * u));
      const float* x = v + 8 * u;
      if constexpr (sizeof(T) == 2) {
        const bf16x8 b = pack8(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, b), p.r, o, 0, kPast);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 y = {x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, y), p.r, o + 16 * h, 0, kPast);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int o = p.at(norm_col<C>(g, 8 * u + e));
        if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (__bf16)v[8 * u + e]), p.r, o, 0, kPast);
        else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v[8 * u + e]), p.r, o, 0, kPast);
      }
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

// x and the lanes it is joined with: DPP inside 16 lanes, swaps of rows of 16 and of halves of the wave beyond
template <int LANES>
__device__ __forceinline__ float lane_sum(float x) {
  auto dpp = [&](auto ctrl) {
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  dpp(std::integral_constant<int, 0xb1>{});         // quad_perm 1, 0, 3, 2
  dpp(std::integral_constant<int, 0x4e>{});         // quad_perm 2, 3, 0, 1
  dpp(std::integral_constant<int, 0x141>{});        // row_half_mirror: the other four of eight
  dpp(std::integral_constant<int, 0x140>{});        // row_mirror: the other eight of sixteen
  if constexpr (LANES > 16) {
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    const auto p = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    x = __builtin_bit_cast(float, (uint32_t)p[0]) + __builtin_bit_cast(float, (uint32_t)p[1]);
  }
  if constexpr (LANES > 32) {
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    const auto p = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    x = __builtin_bit_cast(float, (uint32_t)p[0]) + __builtin_bit_cast(float, (uint32_t)p[1]);
  }
  return x;
}

// N sums over the threads of a row, in every one of them.  s_sum: waves x N floats, another place than that of the call before.
template <class C, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float* s_sum) {
#pragma unroll
  for (int n = 0; n < N; ++n) x[n] = lane_sum<C::LANES>(x[n]);
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
  if (width <= 1536) return f(NormCfg<64, 3, 1, WIDE>{});
  if (width <= 2048) return f(NormCfg<64, 4, 1, WIDE>{});
  if (width <= 4096) return f(NormCfg<256, 2, 2, WIDE>{});
  if (width <= 6144) return f(NormCfg<256, 3, 1, WIDE>{});
  if (width <= 8192) return f(NormCfg<256, 4, 1, WIDE>{});
  if (width <= 12288) return f(NormCfg<512, 3, 1, WIDE>{});
  return f(NormCfg<512, 4, 1, WIDE>{});
}

}  // namespace knap
