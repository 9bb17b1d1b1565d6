// Matrix products of the gated feed-forward block: C[m][n] = sum over k of A(m, k) B(n, k), bf16 operands, 32-bit sums on the matrix cores.
// An operand either lies with k along its rows (ROWK: element (r, k) at r ld + k) or with k down its rows (element (r, k) at k ld + r), so that
// all products of the block take their tensors as they are: nothing is transposed in memory.
//
// A workgroup of WM x WN waves forms a tile of BM x BN, a wave TM x TN blocks of 32 x 32.  Stages of 64 k's go through a ring of two to six buffers in
// LDS, filled past the registers by asynchronous copies: [rows][64] for ROWK, whose rows are whole lines of 128 bytes, read 16 bytes a lane, and [64][128]
// for the other, read transposed, both in layouts that neither way of reading meets a bank twice in.  A wave reads fragments one or two steps of 16 k's
// ahead of their products.  Once a stage's last fragments are asked for, it meets the others: their reads of this buffer are behind them, so that it is
// free for the stage BUFFERS further on, and their copies of the next stage have arrived; and goes on with products of fragments that it has.  The matrix
// cores wait at no barrier for memory.  Waves of 128 x 128 read half as much from LDS as those of 128 x 64 would, two of which share a SIMD (8192^3, us: 823
// and 892, before what the epilogue saves).  The buffers are arrays of their own, and the ring is unrolled: of one array the compiler would wait for every
// copy under way in front of each transposed read (8192^3 with k down the rows of b: 1607 us so, 800 as it is).
//
// Bound by the matrix cores at the clock that the card holds under them: 32768 x 1536 x 4096 takes 310 us (1.33 PFLOP/s; 64 steps of 2.3 to 2.6 thousand
// clocks, of which 2048 are products, at 1.7 GHz).
//
// Rows and k's that a tensor does not have are zeros: the descriptors end behind its last row; k's behind a row's end, which memory
// holds something else at, are asked for behind the descriptor.  Columns behind the last one of a tensor with k down its rows are whatever the next row
// holds; they only meet results that are not stored.
#pragma once

#include "knap_device.h"
#include "knap_kernels.h"

#include <type_traits>
#include <utility>

namespace knap {

constexpr int kGemmK = 64;                // k's of a stage
constexpr int kGemmNowhere = 0x7fffffe0;  // a byte offset behind every descriptor

template <int BM_, int BN_, int WM_, int WN_, int BUFFERS_, int AHEAD_>
struct GemmCfg {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int BUFFERS = BUFFERS_;                // of the ring, 2 to 6
  static constexpr int AHEAD = AHEAD_;                    // steps of 16 k's that fragments are read ahead of their products (1 or 2)
  static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  static constexpr int STAGE = (BM + BN) * kGemmK;      // elements
  static constexpr int LDS_BYTES = BUFFERS * STAGE * 2;
};
struct GemmBuffers { __bf16 *b0, *b1, *b2, *b3, *b4, *b5; };
template <int B>
__device__ __forceinline__ __bf16* buffer_of(const GemmBuffers& s) {
  if constexpr (B == 0) return s.b0;
  else if constexpr (B == 1) return s.b1;
  else if constexpr (B == 2) return s.b2;
  else if constexpr (B == 3) return s.b3;
  else if constexpr (B == 4) return s.b4;
  else return s.b5;
}

// f of 0, 1, ... as types, up to the first that returns false
template <class F, int... B>
__device__ __forceinline__ bool while_true(F& f, std::integer_sequence<int, B...>) { return (f(std::integral_constant<int, B>{}) && ...); }

// Copies of R rows (columns) of an operand for one stage: instruction i of a wave fills 1 KB.
// ROWK: 8 rows of 128 bytes.  Unit c (16 bytes) of row r lies at c ^ ((r / 2) % 8): 16 rows put one unit in 16 places of a 256-byte line.
// else: 4 rows of 256 bytes in one of the R / 128 blocks of [64][128], a Tile<128>.
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

// What the copies of an operand take, stage after stage: the descriptor of this one's k's.
template <bool ROWK>
struct OperandStream {
  uint64_t base, step;      // of the stage's first k; bytes to the next
  uint32_t bytes;           // of the descriptor, but for those that the number of k's decides
  uint32_t ld2;             // bytes of a row
  // rows [first, first + tile) of `limit`, from k0 on
  __device__ __forceinline__ void aim(const __bf16* p, int64_t ld, int first, int limit, int tile, int k0) {
    ld2 = (uint32_t)ld * 2u;
    if constexpr (ROWK) {
      base = reinterpret_cast<uint64_t>(p + (int64_t)first * ld + k0);
      step = 2 * kGemmK;
      bytes = (uint32_t)(min(tile, limit - first) - 1) * ld2;      // up to the last row; its k's are added below
    } else {
      base = reinterpret_cast<uint64_t>(p + (int64_t)k0 * ld + first);
      step = (uint64_t)ld2 * kGemmK;
      bytes = (uint32_t)(limit - first) * 2u;                      // of the last row of the stage; the others are added below
    }
  }
  // `left` k's from here on, none where that is 0 or less
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(int left) const {
    const uint32_t n = (uint32_t)min(left, kGemmK);
    const uint32_t all = ROWK ? bytes + 2 * n : (n - 1) * ld2 + bytes;
    return make_rsrc(reinterpret_cast<const void*>(base), left > 0 ? all : 0u);
  }
};

// The accumulators of one tile (m0, n0), stages [s0, s1) of all segments.
// PAIRED: b of even and of odd blocks of 32 columns are two matrices; TWO: there are two segments.
template <class C, bool A_ROWK, bool B_ROWK, bool PAIRED, bool TWO>
__device__ __forceinline__ void gemm_tile(const GemmProblem& p, int m0, int n0, int s0, int s1, const GemmBuffers& lds, f32x16 (&acc)[C::TM][C::TN]) {
  using LA = OperandLoader<C::BM, A_ROWK, C::WAVES>;
  using LB = OperandLoader<C::BN, B_ROWK, C::WAVES>;
  constexpr int L = LA::COUNT + LB::COUNT, SUB = kGemmK / 16;      // copies of a stage, its steps of 16 k's
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WN, wn = wave % C::WN;
  const int per = (p.K + kGemmK - 1) / kGemmK;      // stages of a segment
#pragma unroll
  for (int i = 0; i < C::TM; ++i)
#pragma unroll
    for (int j = 0; j < C::TN; ++j) acc[i][j] = zero16();
  if (s0 >= s1) return;

  // byte offsets of this lane's 16 bytes from the stage's base
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
  const int columns = min(p.N, n0 + p.step);      // the tile's end
  // the stage that is copied next
  OperandStream<A_ROWK> sa;
  OperandStream<B_ROWK> sb, sb2;
  int at = s0, left;
  auto enter = [&](int seg, int k0) {
    sa.aim(p.a[seg], p.lda, m0, p.M, C::BM, k0);
    sb.aim(p.b[PAIRED ? 0 : seg], p.ldb, n0, columns, PAIRED ? C::BN / 2 : C::BN, k0);
    if constexpr (PAIRED) sb2.aim(p.b[1], p.ldb, n0, columns, C::BN / 2, k0);
    left = p.K - k0;
  };
  const int seg = TWO && s0 >= per ? 1 : 0;
  enter(seg, (s0 - seg * per) * kGemmK);
  auto advance = [&]() {
    ++at;
    sa.base += sa.step;
    sb.base += sb.step;
    if constexpr (PAIRED) sb2.base += sb2.step;
    left -= kGemmK;
    if constexpr (TWO) {
      if (at == per) enter(1, 0);
    }
  };
  // its descriptors; of a stage that there is not they are empty, and its buffer gets zeros, so that waits count alike
  __amdgpu_buffer_rsrc_t da, db, db2;
  int k;
  auto prepare = [&]() {
    k = at < s1 ? left : 0;
    da = sa.descriptor(k);
    db = sb.descriptor(k);
    if constexpr (PAIRED) db2 = sb2.descriptor(k);
  };
  // copies [from, to) of the L
  auto copy = [&](__bf16* buffer, int from, int to) {
#pragma unroll
    for (int q = 0; q < L; ++q) {
      if (q < from || q >= to) continue;
      if (q < LA::COUNT) {
        int o = off_a[q];
        if constexpr (A_ROWK) o = 8 * LA::unit(q, wave, lane) >= k ? kGemmNowhere : o;
        copy_1k(buffer + LA::place(q, wave), da, o);
      } else {
        const int i = q - LA::COUNT;
        int o = off_b[i];
        if constexpr (B_ROWK) o = 8 * LB::unit(i, wave, lane) >= k ? kGemmNowhere : o;
        const bool odd = PAIRED && (LB::row(i, wave, 0) & 32);
        copy_1k(buffer + C::BM * kGemmK + LB::place(i, wave), odd ? db2 : db, o);
      }
    }
  };
  FragmentReader<A_ROWK> ra;
  FragmentReader<B_ROWK> rb;
  ra.init(lane);
  rb.init(lane);
  constexpr int SETS = 2 * C::AHEAD;
  bf16x8 fa[SETS][C::TM], fb[SETS][C::TN];
  auto read = [&](const __bf16* buffer, int kk) {
#pragma unroll
    for (int j = 0; j < C::TN; ++j) fb[kk % SETS][j] = rb.get(buffer + C::BM * kGemmK, wn * C::TN + j, kk);
#pragma unroll
    for (int i = 0; i < C::TM; ++i) fa[kk % SETS][i] = ra.get(buffer, wm * C::TM + i, kk);
  };
  // the first fragments of the next stage stay where they are read, although the loop may end before their use: the compiler would read them behind
  // the branch, in front of the products that need them
  auto hold = [&]() {
#pragma unroll
    for (int kk = 0; kk < C::AHEAD; ++kk) {
#pragma unroll
      for (int i = 0; i < C::TM; ++i) asm volatile("" : "+v"(fa[kk][i]));
#pragma unroll
      for (int j = 0; j < C::TN; ++j) asm volatile("" : "+v"(fb[kk][j]));
    }
  };
  auto multiply = [&](int kk) {
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j) acc[i][j] = mfma32(fb[kk % SETS][j], fa[kk % SETS][i], acc[i][j]);
  };
  // the order of 16 k's: reads of the next fragments and copies spread over the products
  auto order = [&](auto copies) {      // at most so many of those
    constexpr int MF = C::TM * C::TN, READS = C::TM * (A_ROWK ? 1 : 2) + C::TN * (B_ROWK ? 1 : 2), EACH = (READS + MF - 1) / MF;
    constexpr int N = decltype(copies)::value, TOGETHER = (N + MF - 1) / MF, EVERY = N ? MF * TOGETHER / N : MF + 1;
#pragma unroll
    for (int q = 0; q < MF; ++q) {
      KNAP_SGB(KNAP_SG_MFMA, 1);
      if (q * EACH < READS) KNAP_SGB(KNAP_SG_DS_READ, EACH);
      if (N && q % EVERY == 0 && q / EVERY < N) KNAP_SGB(KNAP_SG_VMEM_READ, TOGETHER);
    }
    KNAP_SCHED_FENCE();
  };
  // the copies of a stage go out in shares beside three steps' products, from the step in front of which its buffer becomes free: behind the barrier
  // of the stage that lies there
  constexpr int SHARES = 3, MEET = SUB - C::AHEAD;      // MEET: the step that the waves meet in front of
  auto share = [](int i) { return L * i / SHARES; };
  prepare();
  auto begin = [&](auto which) {
    copy(buffer_of<decltype(which)::value>(lds), 0, L);
    advance();
    prepare();
    return true;
  };
  constexpr auto buffers = std::make_integer_sequence<int, C::BUFFERS>{};
  while_true(begin, buffers);
  wait_vm<(C::BUFFERS - 1) * L>();
  lds_barrier();
#pragma unroll
  for (int kk = 0; kk < C::AHEAD; ++kk) read(buffer_of<0>(lds), kk);
  KNAP_SCHED_FENCE();
  // `behind`: there is a stage in front of this one, whose buffer is being filled
  auto stage = [&](auto which, auto behind) {
    constexpr int B = decltype(which)::value, N = C::BUFFERS;
    constexpr bool FILL = decltype(behind)::value;
#pragma unroll
    for (int kk = 0; kk < SUB; ++kk) {
      if (kk == MEET) {
        wait_vm<(N - 2) * L>();
        lds_barrier();
        KNAP_SCHED_FENCE();
      }
      const int i = kk >= MEET ? kk - MEET : kk + C::AHEAD;      // the share that goes out here
      const bool fill = i < SHARES && (kk >= MEET || FILL);
      if (fill) {
        if (kk >= MEET) copy(buffer_of<B>(lds), share(i), share(i + 1));
        else copy(buffer_of<(B + N - 1) % N>(lds), share(i), share(i + 1));
      }
      if (kk < MEET) read(buffer_of<B>(lds), kk + C::AHEAD);
      else read(buffer_of<(B + 1) % N>(lds), kk - MEET);
      multiply(kk);
      order(std::integral_constant<int, (L + SHARES - 1) / SHARES>{});
      if (fill && i == SHARES - 1) {      // the descriptors of the next stage, beside the products that copy nothing
        advance();
        prepare();
      }
    }
    hold();
  };
  int s = s0;
  stage(std::integral_constant<int, 0>{}, std::false_type{});
  auto go = [&](auto before) {      // the stage behind the one in buffer `before`
    if (++s >= s1) return false;
    stage(std::integral_constant<int, (decltype(before)::value + 1) % C::BUFFERS>{}, std::true_type{});
    return true;
  };
  while (while_true(go, buffers)) {
  }
  wait_vm<0>();
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
