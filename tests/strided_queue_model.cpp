// The device's strided work queue (csrc/knap_strided_queue.h) compiled for the CPU: the same text, with the few device words it uses
// defined here.
#include <algorithm>
#include <vector>

#define __device__
#define __forceinline__ inline
#define __builtin_amdgcn_readfirstlane(x) (x)
using std::max;
using std::min;
static struct { int x; } gridDim, blockIdx;

#include "knap_strided_queue.h"

// lens: the sequences' lengths.  Returns how many items were not dealt exactly once, tickets not served, counters that a last draw does not put
// back, or items out of the list's order; order 0: tile by tile of one sequence after the other, 1: by tiles left.
extern "C" int strided_queue_walk(const int* lens, int n_seq, int H, int tile, int order, int grid) {
  std::vector<int> sorted(lens, lens + n_seq), tiles(n_seq), start(n_seq + 1, 0);
  std::sort(sorted.begin(), sorted.end(), [](int a, int b) { return a > b; });
  for (int r = 0; r < n_seq; ++r) {
    tiles[r] = (sorted[r] + tile - 1) / tile;
    start[r + 1] = start[r] + H * tiles[r];
  }
  const int n = start[n_seq];
  std::vector<int> seen(n, 0);
  std::vector<unsigned> counters(8, 0);
  int wrong = 0, last_left = 1 << 30;
  for (int w = 0; w < n; ++w) {      // the list: every tile once, in order
    const knap::ItemPlace p = order == 0 ? knap::tile_major_item(w, n_seq, H, start.data()) : knap::most_left_item(w, n_seq, H, start.data());
    if (p.rank < 0 || p.rank >= n_seq || p.head < 0 || p.head >= H) { ++wrong; continue; }
    const int at = order == 0 ? p.tile : tiles[p.rank] - p.tile;
    if (at < 0 || at >= tiles[p.rank]) { ++wrong; continue; }
    ++seen[start[p.rank] + p.head * tiles[p.rank] + at];
    if (order == 1) {
      wrong += p.tile > last_left;
      last_left = p.tile;
    }
  }
  for (int w = 0; w < n; ++w) wrong += seen[w] != 1;
  gridDim.x = grid;
  std::vector<int> dealt(n, 0);
  const int n_q = grid % 8 == 0 ? 8 : 1;
  for (int q = 0; q < n_q; ++q) {
    blockIdx.x = q;
    knap::StridedQueue queue;
    queue.init(counters.data(), n);
    wrong += queue.ctr != counters.data() + q || queue.draws != (queue.wide > queue.per);
    for (int i = 0; i < queue.per; ++i) {
      blockIdx.x = q + i * n_q;
      wrong += queue.first_ticket() != i;
    }
    wrong += queue.later_ticket(0u) != queue.per;
    for (int t = 0; t < queue.wide; ++t) {
      const int w = queue.item(t);
      if (w < 0 || w >= n) ++wrong; else ++dealt[w];
    }
    if (queue.draws) {
      int at_work = queue.per;
      for (unsigned drawn = 0; at_work > 0 && drawn <= (unsigned)queue.wide; ++drawn) {
        if (queue.later_ticket(drawn) >= queue.wide) --at_work;
        wrong += queue.last_draw(drawn) != (at_work == 0);
      }
      wrong += at_work != 0;
    }
  }
  for (int w = 0; w < n; ++w) wrong += dealt[w] != 1;
  return wrong;
}
