// Byte offsets of rows that several groups of a wave's lanes share one buffer descriptor for.  Integer arithmetic alone, so that the host
// can walk through it as well (tests/row_span_model.cpp).
#pragma once

#include <cstdint>

namespace knap {

// The offset of a column that the row does not have: behind every descriptor, whose bytes stay below 2^29, with room for the offsets of the
// 32 bytes that a lane accesses from there to be added in a signed int.
constexpr int kNoColumn = 0x7fffffe0;

// rows row0, row0 + 1, ... of which the tensor has `left` more; the group's row is the group-th; `stride` columns apart (at most 2^22)
struct RowSpan {
  uint32_t off, end;      // of the group's row, and behind it; 0 and 0 where the tensor does not have it
  __device__ __forceinline__ RowSpan(int group, int64_t left, int64_t stride, int width, uint32_t size) {
    off = (uint32_t)group * (uint32_t)stride * size;
    end = group < left ? off + (uint32_t)width * size : 0u;
  }
  // bytes of the descriptor of `left` rows
  static __device__ __forceinline__ uint32_t bytes(int64_t left, int64_t stride, int width, uint32_t size) {
    return left > 0 ? (uint32_t)((left - 1) * stride + width) * size : 0u;
  }
  __device__ __forceinline__ int at(uint32_t column_byte) const {
    const uint32_t o = off + column_byte;
    return o < end ? (int)o : kNoColumn;
  }
};

}  // namespace knap
