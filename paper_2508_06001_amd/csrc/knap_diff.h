// Differential attention: what its kernels share.
#pragma once

#include "knap_attn_fwd_part.h"
#include "knap_strided_queue.h"

namespace knap {

template <int D>
struct DiffCfg {
  static constexpr int BM = 128;         // query rows per work item
  static constexpr int BN = 64;          // key/value rows per LDS tile
  static constexpr int KC = D / 16;      // contraction chunks over d, the first half of them of map 1
  static constexpr int DB = D / 32;      // 32-wide blocks of d
  static constexpr int TILE_ELEMS = BN * Tile<D>::LD;
};

// workgroups a CU of the forward and of dQ, which their registers allow
constexpr int diff_workgroups(int d) { return d == 64 ? 3 : 2; }

// One map's softmax of a lane's query: the exponent reference (raw score units), it times c, and this lane's share of the row sum
// (32 of every 64 keys).  The reference moves only when a half tile's probabilities against it are too large, as in the forward of plain
// attention.
struct DiffSoftmax {
  float m_ref = -INFINITY, mc = -INFINITY, l = 0.f;

  // takes in the half whose probabilities sum to `sum` in this lane
  template <int DB>
  __device__ __forceinline__ void settle(const f32x16& s, float c, float sum, bf16x8 (&pb)[2], f32x16 (&o)[DB]) {
    const bool moves = __builtin_amdgcn_ballot_w64(!(sum <= kMaxHalfSum)) != 0;
    if (__builtin_expect(moves, 0)) {
      float m_loc = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) m_loc = fmaxf(m_loc, s[r]);
      const float m_new = fmaxf(m_ref, fmaxf(m_loc, xor32(m_loc)));
      const float alpha = m_new == m_ref ? 1.f : fast_exp2((m_ref - m_new) * c);
      m_ref = m_new;
      mc = m_new == -INFINITY ? 0.f : m_new * c;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
      sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = fast_exp2(__builtin_fmaf(s[r], c, -mc));
        sum += p;
        pb[r >> 3][r & 7] = (__bf16)p;
      }
      if (m_new == -INFINITY) mc = -INFINITY;      // scores of -inf alone set no reference: the next half has to settle too
    }
    l += sum;
    KNAP_SCHED_FENCE();
  }
};

// items of a StridedQueue, whose tiles are of TILE rows
template <int TILE>
__device__ __forceinline__ WorkItem decode_tile_major(int w, const int32_t* __restrict__ cu, int n_seq, int H, const int* s_order, const int* s_start) {
  const ItemPlace p = tile_major_item(w, n_seq, H, s_start);
  WorkItem it = sequence_of_rank(p.rank, cu, s_order);
  it.tile = p.tile;
  it.head = p.head;
  return it;
}
// of which `tile` is the key tile that has as many left, counted from the first, or, FROM_END, the query tile with as many in front of its end
template <int TILE, bool FROM_END>
__device__ __forceinline__ WorkItem decode_most_left(int w, const int32_t* __restrict__ cu, int n_seq, int H, const int* s_order, const int* s_start) {
  const ItemPlace p = most_left_item(w, n_seq, H, s_start);
  WorkItem it = sequence_of_rank(p.rank, cu, s_order);
  it.tile = FROM_END ? p.tile - 1 : (it.len + TILE - 1) / TILE - p.tile;
  it.head = p.head;
  return it;
}

}  // namespace knap
