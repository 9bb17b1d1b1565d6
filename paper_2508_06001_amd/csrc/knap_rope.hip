// Rotary positions of packed queries and keys: the first `rot` columns of every head are pairs, pair i of a row at position p is
// turned by the angle p f_i,
//   (a, b) -> factor (a cos - b sin, a sin + b cos),
// the other columns are copied.  The backward is the transpose: the same with -sin.  A pair's columns are (i, i + rot / 2) in the
// half layout, (2 i, 2 i + 1) in the interleaved one.
//
// What bounds it is HBM: every element is read once and written once, beside 6 flops a pair.  Angles take 64 bits (at position 10^6 a
// 32-bit product is off by 0.06 radians): they are formed once per token and pair, by one thread, reduced to a fraction of a turn
// there, and lie in LDS as (factor cos, factor sin) for all heads of q and k of the workgroup's tokens, so that both go in one launch
// and a 16-byte unit of a row costs 8 LDS pairs and no trigonometry.
#include "knap_device.h"
#include "knap_kernels.h"
#include "knapattn.h"

#include <algorithm>

namespace knap {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxTokens = 8;        // of a workgroup

// number of boundaries of the bag in front of token t, as the first row of its sequence: the largest boundary not behind t; -1 for
// rows at or behind the last boundary, which belong to no sequence.  By one wave.
__device__ __forceinline__ int first_row_of(const int32_t* __restrict__ cu, int n_seq, int t, int lane) {
  int best = 0;
  for (int i = lane; i < n_seq; i += 64) best = max(best, cu[i] <= t ? cu[i] : 0);
  best = __builtin_amdgcn_readlane(wave_max(best), 63);
  return t < cu[n_seq] ? best : -1;
}

__device__ __forceinline__ float lo_of(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float hi_of(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  bf16x2 p;
  p[0] = (__bf16)a;
  p[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, p);
}

// WIDE: every row starts on 16 bytes and no 16-byte unit holds columns of two kinds (rotated first half, second half, copied);
// otherwise pairs and columns are moved one by one.
template <bool HALF, bool WIDE>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  extern __shared__ float2 s_trig[];                 // (tokens, pairs)
  __shared__ int s_first[kRopeMaxTokens];
  const int tid = threadIdx.x, pairs = a.rot / 2;
  const int t0 = (int)blockIdx.x * a.tokens_per_group;
  const int n_tok = min(a.tokens_per_group, a.T - t0);
  if (!a.positions) {
    for (int i = __builtin_amdgcn_readfirstlane(tid >> 6); i < n_tok; i += kRopeThreads / 64) {
      const int first = first_row_of(a.cu, a.n_seq, t0 + i, tid & 63);
      if ((tid & 63) == 0) s_first[i] = first;
    }
    __syncthreads();
  }
  for (int i = tid; i < n_tok * pairs; i += kRopeThreads) {
    const int tok = i / pairs, p = i - tok * pairs;
    int pos;
    if (a.positions) {
      int axis = 0;
#pragma unroll
      for (int x = 0; x < KNAP_ROPE_MAX_AXES - 1; ++x) axis += p >= a.axis_end[x] ? 1 : 0;
      pos = a.positions[(size_t)(t0 + tok) * a.n_axes + min(axis, a.n_axes - 1)];
    } else {
      pos = t0 + tok - s_first[tok];
    }
    double turns = (double)pos * a.freq[p] * 0.15915494309189535;      // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * (float)turns, &s, &c);
    s_trig[i] = make_float2(a.factor * c, a.sign * a.factor * s);
  }
  __syncthreads();

  // slots of a head: units of 8 columns (of the half layout: two of them, a unit and its partner), or single pairs and columns
  const int turned = WIDE ? (HALF ? a.rot / 16 : a.rot / 8) : pairs;
  const int slots = turned + (a.copies ? (WIDE ? (a.d - a.rot) / 8 : a.d - a.rot) : 0);
  const uint32_t per_tok = (uint32_t)(a.H + a.Hk) * (uint32_t)slots;
  for (uint32_t i = tid; i < (uint32_t)n_tok * per_tok; i += kRopeThreads) {
    const uint32_t tok = i / per_tok, rest = i - tok * per_tok, head = rest / (uint32_t)slots;
    const int slot = (int)(rest - head * (uint32_t)slots);
    if (!a.positions && s_first[tok] < 0) continue;
    const bool is_q = head < (uint32_t)a.H;
    const int64_t t = t0 + (int)tok, h = is_q ? head : head - (uint32_t)a.H;
    const __bf16* src = is_q ? a.q + t * a.q_token + h * a.q_head : a.k + t * a.k_token + h * a.k_head;
    __bf16* dst = is_q ? a.q_out + t * a.qo_token + h * a.qo_head : a.k_out + t * a.ko_token + h * a.ko_head;
    const float2* trig = s_trig + (int)tok * pairs;
    if constexpr (WIDE) {
      if (slot >= turned) {
        const int c = a.rot + 8 * (slot - turned);
        *reinterpret_cast<u32x4*>(dst + c) = *reinterpret_cast<const u32x4*>(src + c);
      } else if constexpr (HALF) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(src + 8 * slot), y = *reinterpret_cast<const u32x4*>(src + pairs + 8 * slot);
        u32x4 ox, oy;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 u = trig[8 * slot + 2 * e], v = trig[8 * slot + 2 * e + 1];
          const float a0 = lo_of(x[e]), a1 = hi_of(x[e]), b0 = lo_of(y[e]), b1 = hi_of(y[e]);
          ox[e] = pack2(a0 * u.x - b0 * u.y, a1 * v.x - b1 * v.y);
          oy[e] = pack2(a0 * u.y + b0 * u.x, a1 * v.y + b1 * v.x);
        }
        *reinterpret_cast<u32x4*>(dst + 8 * slot) = ox;
        *reinterpret_cast<u32x4*>(dst + pairs + 8 * slot) = oy;
      } else {
        const u32x4 x = *reinterpret_cast<const u32x4*>(src + 8 * slot);
        u32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 u = trig[4 * slot + e];
          const float a0 = lo_of(x[e]), b0 = hi_of(x[e]);
          o[e] = pack2(a0 * u.x - b0 * u.y, a0 * u.y + b0 * u.x);
        }
        *reinterpret_cast<u32x4*>(dst + 8 * slot) = o;
      }
    } else {
      if (slot >= turned) {
        const int c = a.rot + slot - turned;
        dst[c] = src[c];
      } else {
        const int ca = HALF ? slot : 2 * slot, cb = HALF ? slot + pairs : 2 * slot + 1;
        const float x = (float)src[ca], y = (float)src[cb];
        const float2 u = trig[slot];
        dst[ca] = (__bf16)(x * u.x - y * u.y);
        dst[cb] = (__bf16)(x * u.y + y * u.x);
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(RopeArgs a, bool half, bool wide, int cus, hipStream_t stream) {
  const int turned = wide ? (half ? a.rot / 16 : a.rot / 8) : a.rot / 2;
  const int slots = turned + (a.copies ? (wide ? (a.d - a.rot) / 8 : a.d - a.rot) : 0);
  const int64_t per_tok = (int64_t)(a.H + a.Hk) * slots;
  // tokens of a workgroup: enough slots that its threads have four each, but not so many that the CUs run out of workgroups
  int tokens = (int)std::max<int64_t>(1, std::min<int64_t>(kRopeMaxTokens, 4 * kRopeThreads / per_tok));
  while (tokens > 1 && (a.T + tokens - 1) / tokens < 4 * cus) tokens /= 2;
  a.tokens_per_group = tokens;
  const size_t lds = (size_t)tokens * (a.rot / 2) * sizeof(float2);
  auto* kernel = half ? (wide ? rope_kernel<true, true> : rope_kernel<true, false>) : (wide ? rope_kernel<false, true> : rope_kernel<false, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)((a.T + (int64_t)tokens - 1) / tokens)), dim3(kRopeThreads), lds, stream, a);
  return hipGetLastError();
}

}  // namespace knap
