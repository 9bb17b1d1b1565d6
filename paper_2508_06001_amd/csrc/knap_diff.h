// Differential attention: what its kernels share.
#pragma once

#include "knap_attn_fwd_part.h"

namespace knap {

template <int D>
struct DiffCfg {
  static constexpr int BM = 128;         // query rows per work item
  static constexpr int BN = 64;          // key/value rows per LDS tile
  static constexpr int KC = D / 16;      // contraction chunks over d, the first half of them of map 1
  static constexpr int DB = D / 32;      // 32-wide blocks of d
  static constexpr int TILE_ELEMS = BN * Tile<D>::LD;
};

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

// Every XCD takes every eighth item of the list, in order, its workgroups by drawing from its counter (at zero before the launch).  The
// even queue of plain attention deals out contiguous shares: for the key tiles of two maps, us, shares and this: 17 sequences of 328 .. 4533,
// 24 x 128, under the mask, 2037 and 1707.
struct StridedQueue {
  unsigned* ctr;
  int q, n_q, per, wide;
  bool draws;       // more tickets than workgroups: somebody has to draw
  __device__ __forceinline__ void init(unsigned* counters, int n_items) {
    n_q = (gridDim.x % 8 == 0) ? 8 : 1;
    q = (int)(blockIdx.x % n_q);                  // workgroups go to the XCDs round-robin
    per = (int)gridDim.x / n_q;
    ctr = counters + q;
    wide = __builtin_amdgcn_readfirstlane((n_items - q + n_q - 1) / n_q);
    draws = wide > per;
  }
  __device__ __forceinline__ int first_ticket() const { return (int)blockIdx.x / n_q; }
  __device__ __forceinline__ int later_ticket(unsigned drawn) const { return per + (int)drawn; }
  __device__ __forceinline__ int item(int ticket) const { return q + ticket * n_q; }
  // every workgroup draws until it gets a ticket past the last: `wide` draws in all
  __device__ __forceinline__ bool last_draw(unsigned drawn) const { return drawn + 1 == (unsigned)wide; }
};

// item w of a list that holds, for each sequence, its tiles of TILE rows in turn, and for each of them all heads
template <int TILE>
__device__ __forceinline__ WorkItem decode_tile_major(int w, const int32_t* __restrict__ cu, int n_seq, int H, const int* s_order, const int* s_start) {
  const int r = rank_of_item(s_start, n_seq, w);
  const int rem = w - __builtin_amdgcn_readfirstlane(s_start[r]);
  WorkItem it = sequence_of_rank(r, cu, s_order);
  it.tile = __builtin_amdgcn_readfirstlane(rem / H);
  it.head = __builtin_amdgcn_readfirstlane(rem - it.tile * H);
  return it;
}

// Item w of the list by what is left of the sequence from the tile on, longest first (what a key tile costs under the causal mask): for each
// number c of tiles left, the sequences that have as many, longest first, and for each of them all heads.  Of the tiles with more than n_r
// left (n_r: those of the r-th longest sequence) the first r sequences hold S_r - r n_r, S_r their tiles in all: a search over r finds the n_r
// in front of w, and below it, down to the next one, every c has r + 1 sequences.
template <int TILE>
__device__ __forceinline__ WorkItem decode_most_left(int w, const int32_t* __restrict__ cu, int n_seq, int H, const int* s_order, const int* s_start) {
  auto ahead = [&](int r) { return s_start[r] - r * (s_start[r + 1] - s_start[r]); };      // counted with heads, as s_start is
  int lo = 0, hi = n_seq;        // the last r whose n_r begins at or in front of w
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (ahead(mid) <= w) lo = mid;
    else hi = mid;
  }
  const int r = __builtin_amdgcn_readfirstlane(lo);
  const int at = w - __builtin_amdgcn_readfirstlane(ahead(r)), each = (r + 1) * H;
  const int n_r = __builtin_amdgcn_readfirstlane(s_start[r + 1] - s_start[r]) / H;
  const int left = n_r - at / each, rest = at % each, rank = rest / H;
  WorkItem it = sequence_of_rank(rank, cu, s_order);
  it.head = __builtin_amdgcn_readfirstlane(rest - rank * H);
  it.tile = __builtin_amdgcn_readfirstlane((it.len + TILE - 1) / TILE - left);
  return it;
}

}  // namespace knap
