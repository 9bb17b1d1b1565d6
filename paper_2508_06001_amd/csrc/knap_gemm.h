// Matrix products of the gated feed-forward block: C[m][n] = sum over k of A(m, k) B(n, k), bf16 operands, 32-bit sums on the matrix cores.
// An operand either lies with k along its rows (ROWK: element (r, k) at r ld + k) or with k down its rows (element (r, k) at k ld + r), so that
// all products of the block take their tensors as they are: nothing is transposed in memory.
//
// A workgroup of WM x WN waves forms a tile of BM x BN, a wave TM x TN blocks of 32 x 32.  Steps of 64 k's go through two buffers in LDS,
// filled past the registers by asynchronous copies in the swizzled layouts of knap_device.h: [rows][64] for ROWK, read 16 bytes a lane, and
// [64][128] for the other, read transposed.  A wave reads the fragments of the next 16 k's while it multiplies these; at a step's last 16 it
// first meets the others (whose reads of this step are behind them, so that its buffer is free for the step after next), and goes on with products of
// fragments that it has: the matrix cores wait at no barrier for memory.
//
// Rows and k's that a tensor does not have are zeros: the descriptors end behind its last row; k's behind a row's end, which memory
// holds something else at, are asked for behind the descriptor.  Columns behind the last one of a tensor with k down its rows are whatever the next row
// holds; they only meet results that are not stored.
#pragma once

#include "knap_device.h"
#include "knap_kernels.h"

namespace knap {

constexpr int kGemmK = 64;               // k's of a step
constexpr int kGemmNowhere = 0x7fffffe0;  // a byte offset behind every descriptor

template <int BM_, int BN_, int WM_, int WN_>
struct GemmCfg {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  static constexpr int STAGE = (BM + BN) * kGemmK;      // elements
  static constexpr int LDS_BYTES = 2 * STAGE * 2;
};

// Copies of R rows (columns) of an operand for one step: instruction i of a wave fills 1 KB.
// ROWK: 8 rows of 128 bytes each; else 4 rows of 256 bytes in one of the R / 128 blocks of [64][128].
template <int R, bool ROWK, int WAVES>
struct OperandLoader {
  static constexpr int COUNT = R / 8 / WAVES;
  static_assert(R % (8 * WAVES) == 0 && (ROWK || R % 128 == 0), "whole instructions for every wave");
  // the row (of the R, or of the 64 k's) and the 16-byte unit within it that this lane brings in instruction i
  static __device__ __forceinline__ int row(int i, int wave, int lane) {
    const int q = i * WAVES + wave;
    return ROWK ? 8 * q + (lane >> 3) : 4 * (q & 15) + (lane >> 4);
  }
  static __device__ __forceinline__ int unit(int i, int wave, int lane) {
    const int r = row(i, wave, lane);
    return ROWK ? (lane & 7) ^ ((r >> 1) & 7) : (lane & 15) ^ (4 * (r & 3) + ((r >> 2) & 3));
  }
  static __device__ __forceinline__ int block(int i, int wave) { return ROWK ? 0 : (i * WAVES + wave) >> 4; }
  // LDS element that the instruction starts at
  static __device__ __forceinline__ int place(int i, int wave) { return (i * WAVES + wave) * 512; }
};

__device__ __forceinline__ void copy_1k(__bf16* to, __amdgpu_buffer_rsrc_t r, int offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)to, 16, offset, 0, 0, 0);
}

// Reads of MFMA operands: k's 16 kk + 8 (lane / 32) + 0..7 of row 32 block + lane % 32.
template <bool ROWK>
struct FragmentReader {
  int base;      // bytes
  __device__ __forceinline__ void init(int lane) {
    if constexpr (ROWK) base = 2 * Tile<64>::off(lane & 31, 8 * (lane >> 5));
    else {
      const int i = lane & 15;
      base = 2 * Tile<128>::off(8 * (lane >> 5) + (i >> 2), ((lane >> 4) & 1) * 16 + 4 * (i & 3));
    }
  }
  __device__ __forceinline__ bf16x8 get(const __bf16* tile, int block, int kk) const {
    const char* p = reinterpret_cast<const char*>(tile);
    if constexpr (ROWK) return *reinterpret_cast<const bf16x8*>(p + block * 4096 + (base ^ (32 * kk)));
    else {      // four rows further down the swizzle flips the unit's lowest bit
      const char* q = p + (block >> 2) * 16384 + kk * 4096;
      return join(lds_read_tr(reinterpret_cast<const __bf16*>(q + (base ^ (64 * (block & 3))))),
                  lds_read_tr(reinterpret_cast<const __bf16*>(q + 1024 + (base ^ (64 * (block & 3) + 16)))));
    }
  }
};

// The accumulators of one tile (m0, n0), steps [s0, s1) of all segments.
template <class C, bool A_ROWK, bool B_ROWK, bool PAIRED>
__device__ __forceinline__ void gemm_tile(const GemmProblem& p, int m0, int n0, int s0, int s1, __bf16* lds, f32x16 (&acc)[C::TM][C::TN]) {
  using LA = OperandLoader<C::BM, A_ROWK, C::WAVES>;
  using LB = OperandLoader<C::BN, B_ROWK, C::WAVES>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WN, wn = wave % C::WN;
  const int per = (p.K + kGemmK - 1) / kGemmK;      // steps of a segment
  // byte offsets of this lane's 16 bytes from the step's base, and the k that they start at (ROWK)
  int off_a[LA::COUNT], off_b[LB::COUNT];
#pragma unroll
  for (int i = 0; i < LA::COUNT; ++i)
    off_a[i] = LA::row(i, wave, lane) * (int)p.lda * 2 + LA::block(i, wave) * 256 + LA::unit(i, wave, lane) * 16;
#pragma unroll
  for (int i = 0; i < LB::COUNT; ++i) {
    int r = LB::row(i, wave, lane);
    if constexpr (PAIRED) r = (r >> 6) * 32 + (r & 31);      // which of the two matrices follows from the instruction
    off_b[i] = r * (int)p.ldb * 2 + LB::block(i, wave) * 256 + LB::unit(i, wave, lane) * 16;
  }
  auto copy = [&](int s, int buffer) {
    const int seg = s >= per ? 1 : 0, k0 = (s - seg * per) * kGemmK;
    const bool tail = k0 + kGemmK > p.K;
    __bf16* to_a = lds + buffer * C::STAGE;
    __bf16* to_b = to_a + C::BM * kGemmK;
    auto whole = [&](const __bf16* base, int64_t ld, bool rowk, int first, int limit, int tile) {
      if (rowk) {
        const int64_t rows = min(tile, limit - first);
        return make_rsrc(base + (int64_t)first * ld + k0, rows > 0 ? (uint32_t)((rows * ld - k0) * 2) : 0u);
      }
      const int64_t rows = min(kGemmK, p.K - k0);
      return make_rsrc(base + (int64_t)k0 * ld + first, (uint32_t)(((rows - 1) * ld + limit - first) * 2));
    };
    const __amdgpu_buffer_rsrc_t ra = whole(p.a[seg], p.lda, A_ROWK, m0, p.M, C::BM);
#pragma unroll
    for (int i = 0; i < LA::COUNT; ++i) {
      int o = off_a[i];
      if constexpr (A_ROWK) o = tail && k0 + 8 * LA::unit(i, wave, lane) >= p.K ? kGemmNowhere : o;
      copy_1k(to_a + LA::place(i, wave), ra, o);
    }
    const __amdgpu_buffer_rsrc_t rb0 = whole(p.b[PAIRED ? 0 : seg], p.ldb, B_ROWK, n0, p.N, PAIRED ? C::BN / 2 : C::BN);
    __amdgpu_buffer_rsrc_t rb1 = rb0;
    if constexpr (PAIRED) rb1 = whole(p.b[1], p.ldb, B_ROWK, n0, p.N, C::BN / 2);
#pragma unroll
    for (int i = 0; i < LB::COUNT; ++i) {
      int o = off_b[i];
      if constexpr (B_ROWK) o = tail && k0 + 8 * LB::unit(i, wave, lane) >= p.K ? kGemmNowhere : o;
      const bool odd = PAIRED && (LB::row(i, wave, 0) & 32);
      copy_1k(to_b + LB::place(i, wave), odd ? rb1 : rb0, o);
    }
  };
  FragmentReader<A_ROWK> ra;
  FragmentReader<B_ROWK> rb;
  ra.init(lane);
  rb.init(lane);
  bf16x8 fa[2][C::TM], fb[2][C::TN];
  auto read = [&](int buffer, int kk, int set) {
    const __bf16* ta = lds + buffer * C::STAGE;
    const __bf16* tb = ta + C::BM * kGemmK;
#pragma unroll
    for (int i = 0; i < C::TM; ++i) fa[set][i] = ra.get(ta, wm * C::TM + i, kk);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) fb[set][j] = rb.get(tb, wn * C::TN + j, kk);
  };
#pragma unroll
  for (int i = 0; i < C::TM; ++i)
#pragma unroll
    for (int j = 0; j < C::TN; ++j) acc[i][j] = zero16();
  if (s0 >= s1) return;
  copy(s0, 0);
  if (s0 + 1 < s1) {
    copy(s0 + 1, 1);
    wait_vm<LA::COUNT + LB::COUNT>();
  } else {
    wait_vm<0>();
  }
  lds_barrier();
  read(0, 0, 0);
  int buffer = 0;
  for (int s = s0; s < s1; ++s, buffer ^= 1) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      if (kk < 3) read(buffer, kk + 1, (kk + 1) & 1);
      else if (s + 1 < s1) {
        wait_vm<0>();
        lds_barrier();
        if (s + 2 < s1) copy(s + 2, buffer);
        read(buffer ^ 1, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
#pragma unroll
        for (int i = 0; i < C::TM; ++i) acc[i][j] = mfma32(fb[kk & 1][j], fa[kk & 1][i], acc[i][j]);
    }
  }
  lds_barrier();      // the buffers are free
}

// Where a wave's block (i, j) of a tile lies: this lane's row m, its first column n of unit u (0, 1: columns n .. n + 7)
template <class C>
struct BlockPlace {
  int m, n;
  __device__ __forceinline__ BlockPlace(int m0, int n0, int i, int j) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    m = m0 + (wave / C::WN * C::TM + i) * 32 + (lane & 31);
    n = n0 + (wave % C::WN * C::TN + j) * 32 + 8 * (lane >> 5);
  }
};

// Registers of a block of results <-> 8 consecutive columns a lane.  An accumulator's register r is column 8 (r / 4) + 4 (lane / 32) + r % 4; the lanes
// of a row, l and l ^ 32, trade four columns for each unit.
__device__ __forceinline__ u32x4 pack_unit(const f32x16& x, int u) {
  uint32_t w[2][2];
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      bf16x2 p;
      p[0] = (__bf16)x[8 * u + 4 * g + 2 * i];
      p[1] = (__bf16)x[8 * u + 4 * g + 2 * i + 1];
      w[g][i] = __builtin_bit_cast(uint32_t, p);
    }
  const auto a = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
  const auto b = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
  return u32x4{(uint32_t)a[0], (uint32_t)b[0], (uint32_t)a[1], (uint32_t)b[1]};
}
// the inverse: elements 8 u .. 8 u + 7 of the block's registers
__device__ __forceinline__ void open_unit(u32x4 v, float (&x)[8]) {
  const auto a = __builtin_amdgcn_permlane32_swap((uint32_t)v[0], (uint32_t)v[2], false, false);
  const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)v[1], (uint32_t)v[3], false, false);
  const uint32_t w[4] = {(uint32_t)a[0], (uint32_t)b[0], (uint32_t)a[1], (uint32_t)b[1]};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
  }
}

// a (rows, cols) output or input of the epilogues, from row m0 on
struct TileRows {
  __amdgpu_buffer_rsrc_t r;
  int ld2, m0, cols;
  __device__ __forceinline__ TileRows(const __bf16* base, int64_t ld, int rows, int cols_, int m0_, int tile) : ld2((int)ld * 2), m0(m0_), cols(cols_) {
    const int64_t left = min(tile, rows - m0_);
    r = make_rsrc(base + (int64_t)m0_ * ld, left > 0 ? (uint32_t)(((left - 1) * ld + cols_) * 2) : 0u);
  }
  __device__ __forceinline__ int at(int m, int n) const { return n < cols ? (m - m0) * ld2 + n * 2 : kGemmNowhere; }
  __device__ __forceinline__ void store(int m, int n, u32x4 v) const { __builtin_amdgcn_raw_buffer_store_b128(v, r, at(m, n), 0, 0); }
  __device__ __forceinline__ u32x4 load(int m, int n) const { return __builtin_amdgcn_raw_buffer_load_b128(r, at(m, n), 0, 0); }
};

// Tile t of tiles_m x tiles_n: runs of consecutive tiles take bands of 8 rows of tiles, so that the workgroups that run at one time on an XCD
// (blockIdx % 8) share rows of A and B in its L2.
__device__ __forceinline__ void tile_place(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int band = t / (8 * tiles_n), rest = t - band * 8 * tiles_n;
  const int high = min(8, tiles_m - 8 * band);
  tn = rest / high;
  tm = 8 * band + rest - tn * high;
}
// the place in the order of tiles of workgroup b of n: every XCD takes one run of them
__device__ __forceinline__ int xcd_order(int b, int n) {
  const int xcd = b & 7, i = b >> 3, each = n >> 3, more = n & 7;
  return xcd * each + min(xcd, more) + i;
}

}  // namespace knap
