// Work queue of the kernels of differential attention: a list of items, dearest first, drawn one by one.  Integer arithmetic on the
// schedule alone, so that the host can walk through it as well (tests/strided_queue_model.cpp).
#pragma once

#include "knap_queue.h"

namespace knap {

// Every XCD takes every eighth item of the list, in order, its workgroups by drawing from its counter (at zero before the launch).  The
// even queue of plain attention deals out contiguous shares: for the key tiles of two maps, us, shares and this: 17 sequences of 328 .. 4533,
// 24 x 128, under the mask, 2037 and 1707.  A ticket is drawn at the end of an item: at its start, to hide the draw, the longest items hold the
// next ones (17 of 328 .. 4533, 6 x 128, 505 and 416).
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

struct ItemPlace {
  int rank, head, tile;      // of a sequence by length, of it; `tile` counted as the list says
};

// item w of the list that holds, for each sequence, its tiles in turn, and for each of them all heads
__device__ __forceinline__ ItemPlace tile_major_item(int w, int n_seq, int H, const int* s_start) {
  const int r = __builtin_amdgcn_readfirstlane(rank_of_item(s_start, n_seq, w));
  const int rem = w - __builtin_amdgcn_readfirstlane(s_start[r]);
  const int tile = __builtin_amdgcn_readfirstlane(rem / H);
  return {r, __builtin_amdgcn_readfirstlane(rem - tile * H), tile};
}

// Item w of the list by what is left of the sequence from the tile on, longest first (what a key tile costs under the causal mask, and a query
// tile counted from the end); `tile` here is the number of tiles left.  For each number c of tiles left it holds the sequences that have as
// many, longest first, and for each of them all heads.  Of the tiles with more than n_r left (n_r: the tiles of the r-th longest sequence) the
// first r sequences hold S_r - r n_r, S_r their tiles in all: a search over r finds the n_r in front of w, and from it down to the next one
// every c has r + 1 sequences.
__device__ __forceinline__ ItemPlace most_left_item(int w, int n_seq, int H, const int* s_start) {
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
  const int rest = at % each, rank = __builtin_amdgcn_readfirstlane(rest / H);
  return {rank, __builtin_amdgcn_readfirstlane(rest - rank * H), __builtin_amdgcn_readfirstlane(n_r - at / each)};
}

}  // namespace knap
