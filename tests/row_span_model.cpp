// The offsets of rows that share a descriptor (csrc/knap_row_span.h) compiled for the CPU: the same text, with the device words it uses
// defined here.
#define __device__
#define __forceinline__ inline
#include "knap_row_span.h"

// A wave of rows of `width` columns of `size` bytes, `stride` columns apart, `lanes` lanes of 8 columns each to a row, `groups` rows side by
// side of which the tensor has `left` more.  Returns how many 16-byte accesses leave a signed int, lie in the descriptor but not in
// the lane's own row, or miss a column that is there.
extern "C" int row_span_walk(int lanes, int groups, long left, long stride, int width, int size) {
  int wrong = 0;
  const long there = left < groups ? left : groups, bytes = knap::RowSpan::bytes(there, stride, width, size);
  wrong += bytes != (there > 0 ? ((there - 1) * stride + width) * size : 0) || bytes >= 1L << 31;
  for (int group = 0; group < groups; ++group) {
    const knap::RowSpan span(group, there, stride, width, size);
    for (int lane = 0; lane < lanes; ++lane) {
      const int at = span.at(8 * lane * size);
      for (int h = 0; h < size / 2; ++h) {
        const long o = (long)at + 16 * h, first = (group * stride + 8 * lane) * size + 16 * h;
        const bool has = group < there && 8 * lane < width;
        wrong += o > 0x7fffffffL || (has ? o != first || o + 16 > bytes : o < bytes);
      }
    }
  }
  return wrong;
}
