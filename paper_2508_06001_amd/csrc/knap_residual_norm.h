// Residual norm: what both directions share (the formulas are at the kernels).  A workgroup stays for a run of consecutive rows and walks
// through it in steps that never cross a sequence's end, so that the sequence's gate, scale and shift lie in registers and, backward, its
// gradients add up there.  Rows, loads and sums are those of knap_layer_norm.h.
#pragma once

#include "knap_layer_norm.h"

namespace knap {

// The sequence that row `row` belongs to and the row behind its last one, `limit` at most; the whole wave takes part.  `row` lies below
// cu[n_seq].  64 boundaries at a time, all loads under way at once: a binary search would wait for memory at each of its steps.
__device__ __forceinline__ void sequence_of(const int32_t* cu, int n_seq, int row, int limit, int& seq, int& end) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int s = 0; s < n_seq; s += 64) {
    const int i = s + lane;
    before += __builtin_popcountll(__ballot(i < n_seq && cu[min(i, n_seq - 1) + 1] <= row));
  }
  seq = min(before, n_seq - 1);
  end = min(__builtin_amdgcn_readfirstlane(cu[seq + 1]), limit);
  if (end <= row) end = row + 1;      // boundaries that fall: some rows' results are undefined, but the walk ends
}

// Where a workgroup is: rows [row, end) of sequence seq are next, none once row == limit.
struct RowCursor {
  int row, end, limit, seq;
  __device__ __forceinline__ void enter(const ResidualArgs& a) {
    if (!a.cu) { seq = 0; end = limit; }
    else if (row < limit) sequence_of(a.cu, a.n_seq, row, limit, seq, end);
  }
  __device__ __forceinline__ void start(const ResidualArgs& a, int first, int last) {
    limit = last;
    if (a.cu) limit = min(limit, max(0, __builtin_amdgcn_readfirstlane(a.cu[a.n_seq])));
    row = min(first, limit);
    end = row;
    seq = 0;
    enter(a);
  }
  __device__ __forceinline__ void step(const ResidualArgs& a, int rows) {
    if (end - row > rows) row += rows;
    else { row = end; enter(a); }
  }
};

// alpha gate wp, and (1 + scale) w, of the thread's columns in sequence `seq`; zeros where the row has no such column
template <class C>
__device__ __forceinline__ void load_gate(const ResidualArgs& a, int seq, int g, float (&gz)[C::COLS]) {
  const int size = a.mod_bf16 ? 2 : 4;
  const char* gate = a.gate ? static_cast<const char*>(a.gate) + (int64_t)seq * a.gate_stride * size : nullptr;
  float wp[C::COLS];
  load_weight<C>(gate, a.mod_bf16, 1.f, g, a.width, gz);
  load_weight<C>(a.post_weight, a.w_bf16, 1.f, g, a.width, wp);
#pragma unroll
  for (int i = 0; i < C::COLS; ++i) gz[i] = norm_has<C>(g, i, a.width) && a.f ? a.alpha * gz[i] * wp[i] : 0.f;
}
template <class C>
__device__ __forceinline__ void load_scale(const ResidualArgs& a, int seq, int g, float (&sw)[C::COLS]) {
  const int size = a.mod_bf16 ? 2 : 4;
  const char* scale = a.scale ? static_cast<const char*>(a.scale) + (int64_t)seq * a.mod_stride * size : nullptr;
  float w[C::COLS];
  load_weight<C>(scale, a.mod_bf16, 0.f, g, a.width, sw);
  load_weight<C>(a.weight, a.w_bf16, 1.f, g, a.width, w);
#pragma unroll
  for (int i = 0; i < C::COLS; ++i) sw[i] = norm_has<C>(g, i, a.width) ? (1.f + sw[i]) * w[i] : 0.f;
}

// Which form a width takes: 8 columns of a thread, or 16 of 513 to 1024 aligned ones and of the widest rows, so that up to 8192 columns the vectors of a sequence and its sums
// fit the registers beside the rows (but for 2 to 4 of a backward of single columns in 32 bits with a branch of 16); two rows at a time where that leaves
// registers (single columns, which take a register each: 7584 rows of 1003 in 32 bits, one and two rows, forward 28 and 35 us).
// Beyond 8192 columns they do not fit: 1024 threads have 128 registers each, and a backward spills 72 to 92 of them in 16-byte accesses and 114 to 218
// column by column, a forward up to 7 and 73 to 116.  Inputs in no cache, norms on both sides, forward and backward with its sums: 8000 rows of 5000, bf16, 92 and
// 225 us (3.5 and 2.1 TB/s); 6000 of 9600, bf16, 114 and 990 (4.0 and 0.7); 3000 of 16384, bf16, 96 and 756; 6000 of 9601, 32 bits, no post norm, 543 and 1146.
template <bool WIDE, class F>
hipError_t residual_form(int width, F f) {
  if constexpr (WIDE) {
    if (width <= 128) return f(NormCfg<16, 1, 2, WIDE>{});
    if (width <= 256) return f(NormCfg<32, 1, 2, WIDE>{});
  }
  if (width <= 512) return f(NormCfg<64, 1, WIDE ? 2 : 1, WIDE>{});
  if constexpr (WIDE) {
    if (width <= 1024) return f(NormCfg<64, 2, 1, WIDE>{});
    if (width <= 1536) return f(NormCfg<192, 1, 2, WIDE>{});
  }
  if (width <= 2048) return f(NormCfg<256, 1, WIDE ? 2 : 1, WIDE>{});
  if (width <= 4096) return f(NormCfg<512, 1, 1, WIDE>{});
  if (width <= 8192) return f(NormCfg<1024, 1, 1, WIDE>{});
  return f(NormCfg<1024, 2, 1, WIDE>{});
}
// whether the next rows' loads are under way while these are worked on: where there are registers for both, which 1024 lanes, of rows wider than 4096, do not have
template <class C, class TX>
constexpr bool residual_ahead() { return C::LANES < 1024 && (C::UNITS == 1 || sizeof(TX) == 2); }

// Rows of a workgroup where `most` of them share `rows`: whole passes, but where there are few rows
inline int residual_chunk(int64_t rows, int64_t most, int pass) {
  const int64_t each = (rows + most - 1) / most;
  return (int)(each > pass ? (each + pass - 1) / pass * pass : each > 0 ? each : 1);
}

}  // namespace knap
