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
// workgroups of a launch.  A grid's threads are counted in 32 bits: one of 2^32 and more is taken modulo 2^32, with no error
constexpr int64_t kRopeMostGroups = ((int64_t)1 << 24) - 1;
static_assert(kRopeMostGroups * kRopeThreads < (int64_t)1 << 32, "");

// number of boundaries of the bag in front of token t, as the first row of its sequence: the largest boundary not behind t; -1 for
// rows at or behind the last boundary, which belong to no sequence.  By one wave, which reads all boundaries: 131072 tokens, 48 heads of 128,
// us: 537 for 1 and 536 for 17 sequences, but 881 for 2048 (519 with the positions given).
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

// How columns are moved:
//   kPairs   one pair, or one copied column, at a time: rows that start on 2 bytes only (31464 tokens, 48 heads of 128, us: 330, and 124 on 16 bytes)
//   kStaged  rows on 16 bytes, but units of 8 columns of which some are turned and some not, or whose partners lie across units: rows go
//            through LDS, 16 bytes at a time either way, and are turned there pair by pair (5810 tokens, 16 heads of 64 of which 20
//            columns turn, us: 10.7, and 24 pair by pair from memory)
//   kUnits   units hold columns of one kind (rotated first half, second half, copied), a thread has one; in the half layout its partner is
//            another unit of the row, which the wave's lanes trade, so that every access of a wave is whole rows (196608 tokens, 6 heads of
//            128 of which 64 columns turn, us: 110 (5.5 TB/s), and 127 with both units of a pair in a thread)
// Loads and stores past the caches: 31464 tokens, 48 heads of 128, us: 139 -> 128, now 124 (6.2 TB/s).
enum RopeForm { kPairs, kStaged, kUnits };
constexpr int kStageColumns = 16384;      // of the rows of a turn through LDS

struct RopeRow {
  const __bf16* src;
  __bf16* dst;
};
// row `head` of a token, heads of q in front of those of k.  Both rows are formed and one is taken: a choice between the strides becomes
// loads of kernel arguments that wait for each other (31464 tokens, 48 heads of 128, us: 128 -> 137).
__device__ __forceinline__ RopeRow rope_row(const RopeArgs& a, int64_t t, uint32_t head) {
  const bool is_q = head < (uint32_t)a.H;
  const int64_t hq = head, hk = (int64_t)head - a.H;
  const __bf16 *sq = a.q + t * a.q_token + hq * a.q_head, *sk = a.k + t * a.k_token + hk * a.k_head;
  __bf16 *dq = a.q_out + t * a.qo_token + hq * a.qo_head, *dk = a.k_out + t * a.ko_token + hk * a.ko_head;
  return {is_q ? sq : sk, is_q ? dq : dk};
}

__device__ __forceinline__ u32x4 unit_load(const __bf16* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
__device__ __forceinline__ void unit_store(__bf16* p, u32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p)); }

template <bool HALF, RopeForm FORM>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  extern __shared__ float2 s_trig[];                 // (tokens, pairs)
  __shared__ int s_first[kRopeMaxTokens];
  const int tid = threadIdx.x, pairs = a.rot / 2;
  const int t0 = (a.first_group + (int)blockIdx.x) * a.tokens_per_group;
  const int n_tok = min(a.tokens_per_group, a.T - t0);
  const uint32_t heads = (uint32_t)(a.H + a.Hk);

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

  if constexpr (FORM == kUnits) {
    // A thread keeps its unit and goes from row to row, `side` of them side by side, without a division for each.  HALF: a row's units are
    // a power of two of lanes of one wave.
    const uint32_t units = (uint32_t)a.d / 8, turned = (uint32_t)a.rot / 8, away = turned / 2;
    const uint32_t side = kRopeThreads / units, u = tid % units, rows = (uint32_t)n_tok * heads;
    if (u >= turned && !a.copies) return;
    uint32_t r = tid / units, tok = r / heads, head = r - tok * heads;
    const uint32_t more_tok = side / heads, more_head = side - more_tok * heads;
    if (r >= side) return;
    // (Two, three or six rows' loads in front of their stores: 196608 tokens, 6 heads, us: 110 -> 125, 131, 139.)
    for (; r < rows; r += side, tok += more_tok, head += more_head) {
      if (head >= heads) {
        head -= heads;
        ++tok;
      }
      if (!a.positions && s_first[tok] < 0) continue;
      const RopeRow row = rope_row(a, t0 + (int)tok, head);
      const u32x4 x = unit_load(row.src + 8 * u);
      u32x4 o = x;
      if (u < turned) {
        const float2* trig = s_trig + tok * (uint32_t)pairs;
        if constexpr (HALF) {
          const bool second = u >= away;
          trig += 8 * (second ? u - away : u);
          const int partner = tid + (second ? -(int)away : (int)away);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t y = (uint32_t)__shfl((int)x[e], partner & 63, 64);
            const float2 p = trig[2 * e], q = trig[2 * e + 1];
            const float s0 = second ? p.y : -p.y, s1 = second ? q.y : -q.y;
            o[e] = pack2(lo_of(x[e]) * p.x + lo_of(y) * s0, hi_of(x[e]) * q.x + hi_of(y) * s1);
          }
        } else {
          trig += 4 * u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 p = trig[e];
            const float a0 = lo_of(x[e]), b0 = hi_of(x[e]);
            o[e] = pack2(a0 * p.x - b0 * p.y, a0 * p.y + b0 * p.x);
          }
        }
      }
      unit_store(row.dst + 8 * u, o);
    }
  } else if constexpr (FORM == kStaged) {
    __bf16* stage = reinterpret_cast<__bf16*>(s_trig + n_tok * pairs + (n_tok * pairs & 1));
    const uint32_t n_rows = (uint32_t)n_tok * heads, most = (uint32_t)(kStageColumns / a.d), units = (uint32_t)a.d / 8;
    for (uint32_t r0 = 0; r0 < n_rows; r0 += most) {
      const uint32_t rows = min(most, n_rows - r0);
      auto row_of = [&](uint32_t r) { return rope_row(a, t0 + (int)((r0 + r) / heads), (r0 + r) % heads); };
      for (uint32_t i = tid; i < rows * units; i += kRopeThreads)
        *reinterpret_cast<u32x4*>(stage + 8 * i) = unit_load(row_of(i / units).src + 8 * (i % units));
      __syncthreads();
      for (uint32_t i = tid; i < rows * (uint32_t)pairs; i += kRopeThreads) {
        const uint32_t r = i / (uint32_t)pairs, p = i - r * (uint32_t)pairs;
        __bf16* at = stage + r * (uint32_t)a.d;
        const uint32_t ca = HALF ? p : 2 * p, cb = HALF ? p + (uint32_t)pairs : 2 * p + 1;
        const float x = (float)at[ca], y = (float)at[cb];
        const float2 u = s_trig[((r0 + r) / heads) * (uint32_t)pairs + p];
        at[ca] = (__bf16)(x * u.x - y * u.y);
        at[cb] = (__bf16)(x * u.y + y * u.x);
      }
      __syncthreads();
      for (uint32_t i = tid; i < rows * units; i += kRopeThreads) {
        if (!a.positions && s_first[(r0 + i / units) / heads] < 0) continue;
        unit_store(row_of(i / units).dst + 8 * (i % units), *reinterpret_cast<const u32x4*>(stage + 8 * i));
      }
      __syncthreads();
    }
  } else {
    const int slots = pairs + (a.copies ? a.d - a.rot : 0);      // of a head: pairs, then single columns
    const uint32_t per_tok = heads * (uint32_t)slots, n_slots = (uint32_t)n_tok * per_tok;
    for (uint32_t i = tid; i < n_slots; i += kRopeThreads) {
      const uint32_t tok = i / per_tok, rest = i - tok * per_tok, head = rest / (uint32_t)slots;
      const int at = (int)(rest - head * (uint32_t)slots);
      if (!a.positions && s_first[tok] < 0) continue;
      const RopeRow row = rope_row(a, t0 + (int)tok, head);
      if (at >= pairs) {
        const int c = a.rot + at - pairs;
        row.dst[c] = row.src[c];
      } else {
        const int ca = HALF ? at : 2 * at, cb = HALF ? at + pairs : 2 * at + 1;
        const float x = (float)row.src[ca], y = (float)row.src[cb];
        const float2 u = s_trig[(int)tok * pairs + at];
        row.dst[ca] = (__bf16)(x * u.x - y * u.y);
        row.dst[cb] = (__bf16)(x * u.y + y * u.x);
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(RopeArgs a, bool half, bool aligned, int cus, hipStream_t stream) {
  const int units = a.d / 8;
  const bool whole = half ? a.rot % 16 == 0 && units <= 64 && (units & (units - 1)) == 0 : a.rot % 8 == 0;
  const RopeForm form = !aligned ? kPairs : whole ? kUnits : kStaged;
  const int64_t per_tok = (int64_t)(a.H + a.Hk) * (form == kPairs ? a.d : units);
  // tokens of a workgroup: enough units that its threads have three or four each, but not so many that the CUs run out of workgroups
  int tokens = (int)std::max<int64_t>(1, std::min<int64_t>(kRopeMaxTokens, 4 * kRopeThreads / per_tok));
  while (tokens > 1 && ((int64_t)a.T + tokens - 1) / tokens < 4 * cus) tokens /= 2;
  a.tokens_per_group = tokens;
  size_t lds = (size_t)tokens * (a.rot / 2) * sizeof(float2);
  if (form == kStaged) lds = (lds + 15) / 16 * 16 + kStageColumns * sizeof(__bf16);
  auto* kernel = half ? (form == kUnits ? rope_kernel<true, kUnits> : form == kStaged ? rope_kernel<true, kStaged> : rope_kernel<true, kPairs>)
                      : (form == kUnits ? rope_kernel<false, kUnits> : form == kStaged ? rope_kernel<false, kStaged> : rope_kernel<false, kPairs>);
  const int64_t groups = ((int64_t)a.T + tokens - 1) / tokens;
  for (int64_t first = 0; first < groups; first += kRopeMostGroups) {
    a.first_group = (int)first;
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(groups - first, kRopeMostGroups)), dim3(kRopeThreads), lds, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace knap
