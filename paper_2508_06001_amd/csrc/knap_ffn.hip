// Gated feed-forward block, forward and backward, of T tokens (rows of x), D columns and F hidden ones:
//   a = x Wg^T,  b = x Wu^T,  h = act(a) b,  y = h Wd^T
//   dh = dy Wd,  da = dh b act'(a),  db = dh act(a),  dx = da Wg + db Wu,  dWg = da^T x,  dWu = db^T x,  dWd = dy^T h
// act(a) = a s with s the logistic function of a (SiLU) or of 2 sqrt(2 / pi) (a + 0.044715 a^3) (GELU in its tanh form).
// Five launches of the product of knap_gemm.h.  a and b are formed side by side, blocks of 32 columns of either in turn, so that a wave has both of
// an element and act(a) b is its epilogue; da and db are the epilogue of dh, which never reaches memory; dx adds up two products over k.
// a, b, h, da and db are rounded to 16 bits: h and da, db, formed from 32-bit values, because they are what the matrix cores multiply next, a and b
// because a backward reads them (in 32 bits 515 MB more to write and as many to read at 31464 x 4096).
// Bound by the matrix cores, the epilogue of the hidden gradients by HBM.  31464 tokens, 1536 x 4096, us and TFLOP/s: up 728 (1088), down 329 (1202), hidden
// gradients 503 (787; 1327 MB read, where a, b, dy and Wd are 625, and 516 written), dx 625 (1266), the weights' gradients 911 (1303); 4173 tokens, 2048 x 5504: up 174 (1080), down 97 (975).
#include "knap_gemm.h"

#include <algorithm>

namespace knap {

enum Epilogue { kStore, kActForward, kActBackward };

// s(a) of the activation and, for its slope, the derivative of its argument
__device__ __forceinline__ float logistic(float u) { return __builtin_amdgcn_rcpf(1.f + fast_exp2(-kLog2e * u)); }
__device__ __forceinline__ void activation(float a, bool gelu, float& s, float& du) {
  if (gelu) {
    // beyond 16 the logistic function is 0 or 1 in 32 bits, and a squared may overflow
    const float c = __builtin_fminf(__builtin_fmaxf(a, -16.f), 16.f);
    constexpr float k = 1.5957691216057308f;      // 2 sqrt(2 / pi)
    s = logistic(k * __builtin_fmaf(0.044715f * c, c * c, c));
    du = k * __builtin_fmaf(3.f * 0.044715f * c, c, 1.f);
  } else {
    s = logistic(a);
    du = 1.f;
  }
}

// da and db of an element.  What may be zero is a factor before what may be large: where the activation or its slope vanishes, a du, dh b and dh a may be
// past the range, and infinity times zero is no number.  Half of the slope, which may be above one, so that b times it stays in the range as well.
__device__ __forceinline__ void hidden_gradient(float dh, float a, float b, bool gelu, float& da, float& db) {
  float s, du;
  activation(a, gelu, s, du);
  const float half = 0.5f * s;
  da = 2.f * (dh * (b * __builtin_fmaf(a * (half * (1.f - s)), du, half)));
  db = dh * (a * s);
}

// The epilogue of one block, from its registers (of tiles whose parts were added up)
template <class C, int EP>
__device__ __forceinline__ void finish_block(const GemmLaunch& g, const GemmProblem& p, int m0, int n0, int i, int j, const f32x16& x, const f32x16& x2) {
  const int columns = min(p.N, n0 + p.step);
  if constexpr (EP == kStore) {
    const BlockPlace<C> at(m0, n0, i, j);
    const TileRows c(p.c, p.ldc, p.M, columns, m0, C::BM);
#pragma unroll
    for (int u = 0; u < 2; ++u) c.store(at.m, at.n + 16 * u, pack_unit(x, u));
  } else if constexpr (EP == kActForward) {      // x, x2: a and b of block j / 2 of the tile's hidden columns
    const BlockPlace<C> pair(m0, 0, i, j);
    const int m = pair.m, wn_first = pair.n - 8 * ((threadIdx.x & 63) >> 5);
    const int n = n0 + wn_first / 2 + 8 * ((threadIdx.x & 63) >> 5);
    f32x16 h;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float s, du;
      activation(x[r], g.gelu, s, du);
      h[r] = x[r] * s * x2[r];
    }
    const TileRows c(g.h, p.N, p.M, columns, m0, C::BM);
#pragma unroll
    for (int u = 0; u < 2; ++u) c.store(m, n + 16 * u, pack_unit(h, u));
    if (g.gate) {
      const TileRows ga(g.gate, p.N, p.M, columns, m0, C::BM), up(g.up, p.N, p.M, columns, m0, C::BM);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        ga.store(m, n + 16 * u, pack_unit(x, u));
        up.store(m, n + 16 * u, pack_unit(x2, u));
      }
    }
  } else {
    const BlockPlace<C> at(m0, n0, i, j);
    const TileRows gi(g.gate_in, p.N, p.M, columns, m0, C::BM), ui(g.up_in, p.N, p.M, columns, m0, C::BM);
    const TileRows go(g.gate, p.N, p.M, columns, m0, C::BM), uo(g.up, p.N, p.M, columns, m0, C::BM);
    f32x16 da, db;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float a[8], b[8];
      open_unit(gi.load(at.m, at.n + 16 * u), a);
      open_unit(ui.load(at.m, at.n + 16 * u), b);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float ga, gb;
        hidden_gradient(x[8 * u + e], a[e], b[e], g.gelu, ga, gb);
        da[8 * u + e] = ga;
        db[8 * u + e] = gb;
      }
      go.store(at.m, at.n + 16 * u, pack_unit(da, u));
      uo.store(at.m, at.n + 16 * u, pack_unit(db, u));
    }
  }
}

// The epilogue of a whole tile.  A wave's rows of results lie across its lanes' registers, so that stores from there would write 32 bytes of 32 rows
// each; they go through its own part of the buffers in LDS, 32 rows at a time, and out in rows, past the caches: what is written there would only
// push out what the other workgroups multiply (256 x 256 tiles, us, from registers, through LDS, and past the caches as well: 32768 x 8192 x 1536
// 809, 741, 640; 8192^3 858, 811, 756).  What the next launch reads, h, da and db, goes through them where it fits into the last one (4173 tokens, 2048 x 5504,
// us of a forward past the caches and through them: 293 and 283, 613 tokens, 1000 x 2664, both directions 93.0 and 89.9; of 31464, 1536 x 4096, where h does
// not fit, 3140 and 3165).
constexpr int kPast = 2;      // the non-temporal bit of a buffer access
template <class C, int EP>
__device__ __forceinline__ void finish_tile(const GemmLaunch& g, const GemmProblem& p, int m0, int n0, const f32x16 (&acc)[C::TM][C::TN],
                                            const GemmBuffers& lds) {
  static_assert((C::WAVES == 4 || C::WAVES <= 2) && C::STAGE >= C::WAVES * 32 * 32 * C::TN, "a wave has half of a buffer, one of two a whole one");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WN, wn = wave % C::WN;
  // (of the LDS address space, which a choice between two arrays otherwise loses)
  using LdsFloat = __attribute__((address_space(3))) float;
  using LdsFloat4 = __attribute__((address_space(3))) f32x4;
  LdsFloat* const part0 = (LdsFloat*)lds.b0;
  LdsFloat* const part1 = (LdsFloat*)lds.b1;
  LdsFloat* mine = (wave & 1 ? part1 : part0) + (wave >> 1) * (C::STAGE / 4);
  constexpr int COLS = 32 * C::TN, UNITS = COLS / 8;      // of a wave's rows
  constexpr int OUT = EP == kActForward ? COLS / 2 : COLS, OUT_UNITS = OUT / 8;      // of an output
  const int n_first = n0 + wn * OUT;
  auto place = [&](int row, int unit) { return mine + row * COLS + (unit ^ (row & (UNITS - 1))) * 8; };
  auto settle = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    KNAP_SCHED_FENCE();
  };
  auto fetch = [&](int row, int unit, float (&v)[8]) {
    const f32x4 x = *(const LdsFloat4*)place(row, unit), y = *(const LdsFloat4*)(place(row, unit) + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = x[e]; v[4 + e] = y[e]; }
  };
  auto put = [&](const TileRows& to, int at, const float (&v)[8]) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, pack8(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7])), to.r, at, 0, kPast);
  };
  const int columns = min(p.N, n0 + p.step);
  auto pass_on = [&](const TileRows& to, int at, const float (&v)[8]) {      // to the next launch
    if (g.keep) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, pack8(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7])), to.r, at, 0, 0);
    else put(to, at, v);
  };
  const TileRows out0(EP == kStore ? p.c : g.gate, EP == kStore ? p.ldc : p.N, g.gate || EP == kStore ? p.M : 0, columns, m0, C::BM);
  const TileRows out1(EP == kStore ? nullptr : g.up, p.N, EP != kStore && g.up ? p.M : 0, columns, m0, C::BM);
  const TileRows in0(EP == kActForward ? g.h : g.gate_in, p.N, p.M, columns, m0, C::BM), in1(g.up_in, p.N, p.M, columns, m0, C::BM);
  constexpr int TURNS = 32 * OUT_UNITS / 64;
  // a and b of 32 rows, asked for while the 32 before them are worked on
  constexpr bool INPUTS = EP == kActBackward;
  u32x4 a_ahead[INPUTS ? TURNS : 1], b_ahead[INPUTS ? TURNS : 1];
  auto ask = [&](int i) {
    if constexpr (INPUTS) {
#pragma unroll
      for (int q = 0; q < TURNS; ++q) {
        const int row = (q * 64 + lane) / OUT_UNITS, unit = (q * 64 + lane) % OUT_UNITS;
        const int at = in0.at(m0 + (wm * C::TM + i) * 32 + row, n_first + 8 * unit);
        a_ahead[q] = __builtin_amdgcn_raw_buffer_load_b128(in0.r, at, 0, kPast);
        b_ahead[q] = __builtin_amdgcn_raw_buffer_load_b128(in1.r, at, 0, kPast);
      }
    }
  };
  ask(0);
#pragma unroll
  for (int i = 0; i < C::TM; ++i) {
    u32x4 a_now[INPUTS ? TURNS : 1], b_now[INPUTS ? TURNS : 1];
    if constexpr (INPUTS) {
#pragma unroll
      for (int q = 0; q < TURNS; ++q) { a_now[q] = a_ahead[q]; b_now[q] = b_ahead[q]; }
      if (i + 1 < C::TM) ask(i + 1);
    }
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)      // columns 8 q + 4 (lane / 32) .. + 3 of the block
        *(LdsFloat4*)(place(lane & 31, 4 * j + q) + 4 * (lane >> 5)) =
            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    settle();
#pragma unroll
    for (int q = 0; q < TURNS; ++q) {
      const int row = (q * 64 + lane) / OUT_UNITS, unit = (q * 64 + lane) % OUT_UNITS;
      const int at = out0.at(m0 + (wm * C::TM + i) * 32 + row, n_first + 8 * unit);
      float x[8];
      if constexpr (EP == kStore) {
        fetch(row, unit, x);
        put(out0, at, x);
      } else if constexpr (EP == kActForward) {
        float b[8], h[8];
        const int from = (unit >> 2) * 8 + (unit & 3);      // a's block of 32 columns, b's behind it
        fetch(row, from, x);
        fetch(row, from + 4, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float s, du;
          activation(x[e], g.gelu, s, du);
          h[e] = x[e] * s * b[e];
        }
        const int place_h = in0.at(m0 + (wm * C::TM + i) * 32 + row, n_first + 8 * unit);
        pass_on(in0, place_h, h);
        put(out0, at, x);
        put(out1, at, b);
      } else {
        const u32x4 av = a_now[q], bv = b_now[q];
        fetch(row, unit, x);
        float da[8], db[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float a = __builtin_bit_cast(float, (e & 1) ? av[e >> 1] & 0xffff0000u : av[e >> 1] << 16);
          const float b = __builtin_bit_cast(float, (e & 1) ? bv[e >> 1] & 0xffff0000u : bv[e >> 1] << 16);
          hidden_gradient(x[e], a, b, g.gelu, da[e], db[e]);
        }
        pass_on(out0, at, da);
        pass_on(out1, at, db);
      }
    }
    settle();
  }
}

// which product a tile is of, and where it lies
template <class C>
__device__ __forceinline__ int locate(const GemmLaunch& g, int tile, int& m0, int& n0) {
  const int q = tile >= g.first[1] ? (tile >= g.first[2] ? 2 : 1) : 0;
  int tm, tn;
  tile_place(tile - g.first[q], g.p[q].tiles_m, g.p[q].tiles_n, tm, tn);
  m0 = tm * C::BM;
  n0 = tn * g.p[q].step;
  return q;
}

template <class C, bool A_ROWK, bool B_ROWK, int EP>
__global__ __launch_bounds__(C::THREADS, C::LDS_BYTES > 81920 || C::WAVES == 1 ? (C::WAVES + 3) / 4 : C::WAVES / 2) void gemm_kernel(GemmLaunch g) {
  __shared__ __align__(1024) __bf16 b0[C::STAGE], b1[C::STAGE], b2[C::BUFFERS > 2 ? C::STAGE : 8], b3[C::BUFFERS > 3 ? C::STAGE : 8],
      b4[C::BUFFERS > 4 ? C::STAGE : 8], b5[C::BUFFERS > 5 ? C::STAGE : 8];
  constexpr bool PAIRED = EP == kActForward, TWO = EP == kStore && A_ROWK && !B_ROWK;      // dx alone adds up two products
  int tile, part = 0, parts = 1;
  if ((int)blockIdx.x < g.whole) tile = xcd_order(blockIdx.x, g.whole);
  else {
    const int r = (int)blockIdx.x - g.whole;
    tile = g.whole + r / g.splits;
    part = r % g.splits;
    parts = g.splits;
  }
  int m0, n0;
  const int q = locate<C>(g, tile, m0, n0);
  const GemmProblem& p = g.p[q];
  const int stages = (p.K + kGemmK - 1) / kGemmK * p.segments;
  f32x16 acc[C::TM][C::TN];
  gemm_tile<C, A_ROWK, B_ROWK, PAIRED, TWO>(p, m0, n0, (int)((int64_t)stages * part / parts), (int)((int64_t)stages * (part + 1) / parts), GemmBuffers{b0, b1, b2, b3, b4, b5}, acc);
  if (parts > 1) {
    f32x4* to = reinterpret_cast<f32x4*>(g.partial) + (size_t)((int)blockIdx.x - g.whole) * (C::BM * C::BN / 4) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          to[((i * C::TN + j) * 4 + k) * C::THREADS] = f32x4{acc[i][j][4 * k], acc[i][j][4 * k + 1], acc[i][j][4 * k + 2], acc[i][j][4 * k + 3]};
    return;
  }
  finish_tile<C, EP>(g, p, m0, n0, acc, GemmBuffers{b0, b1, b2, b3, b4, b5});
}

// Adds up the parts of a tile's block (blockIdx.y; of a pair of blocks) in their order and finishes it
template <class C, int EP>
__global__ __launch_bounds__(C::THREADS) void gemm_join_kernel(GemmLaunch g) {
  constexpr bool PAIRED = EP == kActForward;
  constexpr int STEP = PAIRED ? 2 : 1;
  int m0, n0;
  const int q = locate<C>(g, g.whole + (int)blockIdx.x, m0, n0);
  const int i = (int)blockIdx.y / (C::TN / STEP), j = (int)blockIdx.y % (C::TN / STEP) * STEP;
  f32x16 x[STEP];
  for (int e = 0; e < STEP; ++e) x[e] = zero16();
  for (int z = 0; z < g.splits; ++z) {
    const f32x4* from = reinterpret_cast<const f32x4*>(g.partial) + ((size_t)blockIdx.x * g.splits + z) * (C::BM * C::BN / 4) + threadIdx.x;
#pragma unroll
    for (int e = 0; e < STEP; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x4 v = from[((i * C::TN + j + e) * 4 + k) * C::THREADS];
#pragma unroll
        for (int w = 0; w < 4; ++w) x[e][4 * k + w] += v[w];
      }
  }
  // the block's place is a constant of the epilogue's accesses only by its row and column
#pragma unroll
  for (int ii = 0; ii < C::TM; ++ii)
#pragma unroll
    for (int jj = 0; jj < C::TN; jj += STEP)
      if (ii == i && jj == j) finish_block<C, EP>(g, g.p[q], m0, n0, ii, jj, x[0], x[STEP - 1]);
}

// Forms.  Large: the fewest bytes of LDS and L2 a product; Small: two workgroups a CU; Deep: one, whose copies run four stages ahead, for calls with so
// few tiles that a stage waits for memory (613 tokens, 1000 x 2664, dx without parts: 48 us, Small 70; 4173 tokens, 2048 x 5504, up: Large 167, Small 205,
// Deep 237).
// Large reads its fragments two steps ahead, but for a and b together (4173 tokens, 2048 x 5504, us, two and one: up 181 and 167; 31464 tokens,
// 1536 x 4096: dx 643 and 709, down 299 and 307, up 706 and 691).
template <int EP>
using Large = GemmCfg<256, 256, 2, 2, 2, EP == kActForward ? 1 : 2>;
using Small = GemmCfg<128, 128, 2, 2, 2, 1>;
using Deep = GemmCfg<128, 128, 2, 2, 4, 1>;

// Forms of a row of tiles, for a forward of up to 32 and of up to 64 tokens, bound by the weights' bytes: two workgroups a CU, rings so deep that both have 80 KB
// on the way, and tiles of as many columns, up to 64, as spread them evenly over the CUs.  us of a forward on weights that are in no cache, these forms and
// those above (where the weights lie in memory makes 3 % between two runs): 4096 x 10944, 24 tokens 70 and 79, 48 tokens 73 and 81; 4096 x 16384, 24 tokens 103
// and 110, 48 tokens 104 and 112; 2048 x 5504, 32 tokens 34 and 38, 48 tokens 33 and 41; 768 x 2048, 48 tokens 20 and 23.  128 columns and one workgroup a CU:
// 24 tokens 4096 x 10944 65 to 68, 4096 x 16384 108 to 112, 2048 x 5504 35; 48 tokens 71, 109, 38.
using Few32 = GemmCfg<32, 64, 1, 1, 6, 1>;
using Few64 = GemmCfg<64, 64, 2, 1, 5, 1>;

// ---------------------------------------------------------------------------
// Plans
// ---------------------------------------------------------------------------
// The card's, not asked of the device: a call's plan, and with it the size of its workspace, depends on its sizes alone.  On a device of other compute units (a
// partition) results are as right, and the last round of tiles is cut for another one.
constexpr int kGemmCus = 256;

// What a form costs, in us, as measured: a stage of a round of workgroups with `fill` of the card's places taken, and what a part adds that is written
// and read again.  It compares forms of many stages.  A launch's start, a ring's first fill and the epilogue are not in it: calls of few stages take about
// twice as long (613 tokens, 1000 x 2664, 16 stages: up 9.0 by it and 16.4 us, hidden gradients 7.5 and 19.4).
struct FormCost {
  int places;                   // workgroups at one time
  float stage, more, part;      // a stage takes stage + more * fill
};
template <class C> constexpr FormCost form_cost() { return {kGemmCus, 1.15f, 0.55f, 0.105f}; }      // Large
template <> constexpr FormCost form_cost<Small>() { return {2 * kGemmCus, 0.62f, 0.43f, 0.026f}; }
template <> constexpr FormCost form_cost<Deep>() { return {kGemmCus, 0.38f, 0.22f, 0.026f}; }
constexpr float kJoin = 4.f;      // the launch that adds up parts (4.8 to 6.6 us of few, 12.6 of the weights' gradients of 1536 x 4096)

// Lays down the tiles of the products in `g` in form C, and how many parts the tiles of the last round go in (which is not full: more of them take less
// time and more bytes); returns the estimated time.
template <class C>
float plan(GemmLaunch& g, bool paired) {
  int tiles = 0, stages = 1 << 30;
  for (int q = 0; q < 3; ++q) {
    g.first[q] = q < g.n ? tiles : INT32_MAX;
    if (q >= g.n) continue;
    GemmProblem& p = g.p[q];
    const int bn = paired ? C::BN / 2 : C::BN;
    p.tiles_m = (p.M + C::BM - 1) / C::BM;
    p.tiles_n = (p.N + bn - 1) / bn;
    p.step = bn;
    tiles += p.tiles_m * p.tiles_n;
    stages = std::min(stages, (p.K + kGemmK - 1) / kGemmK * p.segments);
  }
  constexpr FormCost f = form_cost<C>();
  const int rest = tiles % f.places;
  float last = 0.f;
  g.splits = 1;
  if (rest) {
    auto round = [&](int parts) { return (float)stages / (float)parts * (f.stage + f.more * (float)(rest * parts) / (float)f.places); };
    last = round(1);
    const int most = std::min(f.places / rest, stages / 4);
    for (int parts = 2; parts <= most; ++parts) {
      const float t = round(parts) + kJoin + f.part * (float)(rest * parts);
      if (t < last) { last = t; g.splits = parts; }
    }
  }
  g.whole = g.splits > 1 ? tiles - rest : tiles;
  g.tail = tiles - g.whole;
  return (float)(tiles / f.places) * (float)stages * (f.stage + f.more) + last;
}

// The same for one product of one row of tiles in a form for few tokens: how many columns a tile has, and how many parts it goes in.
template <class C>
void plan_few(GemmLaunch& g, bool paired) {
  // us: a launch's start, a stage at least, a row of 128 bytes that a CU reads, a part that is written and read again
  constexpr float kStart = 3.f, kStage = 0.35f, kRow = 0.0046f, kPart = 0.5f * C::BM * C::BN * 1e-6f;
  static_assert(C::LDS_BYTES <= 81920, "two workgroups a CU");
  constexpr int PLACES = 2;      // of a CU
  GemmProblem& p = g.p[0];
  const int mats = paired ? 2 : 1, stages = (p.K + kGemmK - 1) / kGemmK;
  float best = 1e30f;
  for (int step = 8; step <= C::BN / mats && step < p.N + 8; step += 8) {
    const int tiles = (p.N + step - 1) / step;
    const float row = kRow * (float)(mats * step + p.M);
    for (int parts = 1; parts == 1 || (tiles * parts <= PLACES * kGemmCus && parts <= stages / 4); ++parts) {
      const int each = (tiles * parts + kGemmCus - 1) / kGemmCus;      // workgroups of a CU
      const float rounds = (float)((each + PLACES - 1) / PLACES);
      float t = rounds * kStart + (float)stages / (float)parts * std::max(rounds * kStage, (float)each * row);
      if (parts > 1) t += kJoin + kPart * (float)(tiles * parts);
      if (t >= best) continue;
      best = t;
      p.step = step;
      p.tiles_n = tiles;
      g.splits = parts;
    }
  }
  p.tiles_m = 1;
  g.first[0] = 0;
  g.first[1] = g.first[2] = INT32_MAX;
  g.whole = g.splits > 1 ? 0 : p.tiles_n;
  g.tail = p.tiles_n - g.whole;
}

template <class C>
size_t parts_bytes(const GemmLaunch& g) { return (size_t)g.tail * g.splits * C::BM * C::BN * sizeof(float); }

// calls f(form, launch) with the form of the least estimated time.  ROWS: both operands have k along their rows, as in a forward
template <int EP, bool ROWS, class F>
auto with_form(const GemmLaunch& g, F f) {
  constexpr bool paired = EP == kActForward;
  if constexpr (ROWS) {
    GemmLaunch few = g;
    if (g.p[0].M <= 32) {
      plan_few<Few32>(few, paired);
      return f(Few32{}, few);
    }
    if (g.p[0].M <= 64) {
      plan_few<Few64>(few, paired);
      return f(Few64{}, few);
    }
  }
  GemmLaunch large = g, small = g, deep = g;
  const float tl = plan<Large<EP>>(large, paired), ts = plan<Small>(small, paired), td = plan<Deep>(deep, paired);
  if (tl <= ts && tl <= td) return f(Large<EP>{}, large);
  if (ts <= td) return f(Small{}, small);
  return f(Deep{}, deep);
}

template <class C, bool A_ROWK, bool B_ROWK, int EP>
hipError_t launch_gemm(const GemmLaunch& g, hipStream_t stream) {
  constexpr int BLOCKS = C::TM * C::TN / (EP == kActForward ? 2 : 1);
  // A grid has fewer than 2^32 threads: 2^24 workgroups of 256.  The entry points let up to 2^37 results of a product pass, which are at most 2^22 + 2^18 + 2^9
  // of Large's tiles.  The other forms' tiles are a quarter of those, but a form is taken by its estimate, which for many tiles is 1.7 / 256 a tile of Large,
  // 1.05 / 512 of Small and 0.6 / 256 of Deep: where there are more than 3.3 times as many of them, Large is taken.
  if (g.whole + (int64_t)g.tail * g.splits >= 1 << 24) return hipErrorInvalidValue;
  hipLaunchKernelGGL((gemm_kernel<C, A_ROWK, B_ROWK, EP>), dim3(g.whole + g.tail * g.splits), dim3(C::THREADS), 0, stream, g);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.tail == 0) return e;
  hipLaunchKernelGGL((gemm_join_kernel<C, EP>), dim3(g.tail, BLOCKS), dim3(C::THREADS), 0, stream, g);
  return hipGetLastError();
}

template <int EP, bool ROWS = false>
size_t bytes_of(const GemmLaunch& g) {
  return with_form<EP, ROWS>(g, [](auto form, const GemmLaunch& planned) { return parts_bytes<decltype(form)>(planned); });
}
template <bool A_ROWK, bool B_ROWK, int EP>
hipError_t run(const GemmLaunch& g, hipStream_t stream) {
  return with_form<EP, A_ROWK && B_ROWK>(g, [&](auto form, const GemmLaunch& planned) { return launch_gemm<decltype(form), A_ROWK, B_ROWK, EP>(planned, stream); });
}

constexpr int64_t kKeptBytes = 128 << 20;      // half of the card's last cache

static GemmProblem product(const __bf16* a, int64_t lda, const __bf16* b, int64_t ldb, __bf16* c, int64_t ldc, int M, int N, int K) {
  GemmProblem p{};
  p.a[0] = p.a[1] = a;
  p.b[0] = p.b[1] = b;
  p.c = c;
  p.lda = lda; p.ldb = ldb; p.ldc = ldc;
  p.M = M; p.N = N; p.K = K;
  p.segments = 1;
  return p;
}

static GemmLaunch up_products(const FfnArgs& a) {
  GemmLaunch g{};
  g.n = 1;
  g.p[0] = product(a.x, a.x_stride, a.w_gate, a.width, nullptr, 0, a.tokens, a.hidden, a.width);
  g.p[0].b[1] = a.w_up;
  g.gate = a.gate; g.up = a.up; g.h = a.h;
  g.keep = (int64_t)a.tokens * a.hidden * 2 <= kKeptBytes;
  g.gelu = a.gelu;
  g.partial = a.partial;
  return g;
}
static GemmLaunch down_product(const FfnArgs& a) {
  GemmLaunch g{};
  g.n = 1;
  g.p[0] = product(a.h, a.hidden, a.w_down, a.hidden, a.y, a.y_stride, a.tokens, a.width, a.hidden);
  g.partial = a.partial;
  return g;
}
static GemmLaunch hidden_gradients(const FfnArgs& a) {
  GemmLaunch g{};
  g.n = 1;
  g.p[0] = product(a.dy, a.dy_stride, a.w_down, a.hidden, nullptr, 0, a.tokens, a.hidden, a.width);
  g.gate_in = a.gate; g.up_in = a.up;
  g.gate = a.dgate; g.up = a.dup;
  g.keep = (int64_t)a.tokens * a.hidden * 4 <= kKeptBytes;
  g.gelu = a.gelu;
  g.partial = a.partial;
  return g;
}
static GemmLaunch input_gradient(const FfnArgs& a) {
  GemmLaunch g{};
  g.n = 1;
  g.p[0] = product(a.dgate, a.hidden, a.w_gate, a.width, a.dx, a.dx_stride, a.tokens, a.width, a.hidden);
  g.p[0].a[1] = a.dup;
  g.p[0].b[1] = a.w_up;
  g.p[0].segments = 2;
  g.partial = a.partial;
  return g;
}
static GemmLaunch weight_gradients(const FfnArgs& a) {
  GemmLaunch g{};
  if (a.dw_gate) g.p[g.n++] = product(a.dgate, a.hidden, a.x, a.x_stride, a.dw_gate, a.width, a.hidden, a.width, a.tokens);
  if (a.dw_up) g.p[g.n++] = product(a.dup, a.hidden, a.x, a.x_stride, a.dw_up, a.width, a.hidden, a.width, a.tokens);
  if (a.dw_down) g.p[g.n++] = product(a.dy, a.dy_stride, a.h, a.hidden, a.dw_down, a.hidden, a.width, a.hidden, a.tokens);
  g.partial = a.partial;
  return g;
}

size_t ffn_partial_bytes(int64_t tokens, int width, int hidden, bool backward) {
  FfnArgs a{};
  a.tokens = (int)tokens; a.width = width; a.hidden = hidden;
  if (!backward && ffn_few(tokens, width, hidden)) return 0;
  if (!backward) return std::max(bytes_of<kActForward, true>(up_products(a)), bytes_of<kStore, true>(down_product(a)));
  size_t most = std::max(bytes_of<kActBackward>(hidden_gradients(a)), bytes_of<kStore>(input_gradient(a)));
  __bf16* const some = reinterpret_cast<__bf16*>(16);      // asked for, not looked at
  for (int wanted = 1; wanted < 8; ++wanted) {             // whichever gradients of weights a call wants
    a.dw_gate = wanted & 1 ? some : nullptr;
    a.dw_up = wanted & 2 ? some : nullptr;
    a.dw_down = wanted & 4 ? some : nullptr;
    most = std::max(most, bytes_of<kStore>(weight_gradients(a)));
  }
  return most;
}

hipError_t launch_ffn_fwd(const FfnArgs& a, hipStream_t stream) {
  if (ffn_few(a.tokens, a.width, a.hidden)) return launch_ffn_few(a, stream);
  const hipError_t e = run<true, true, kActForward>(up_products(a), stream);
  return e != hipSuccess ? e : run<true, true, kStore>(down_product(a), stream);
}

hipError_t launch_ffn_bwd(const FfnArgs& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.tokens > 0 && (a.dx || a.dw_gate || a.dw_up)) e = run<true, false, kActBackward>(hidden_gradients(a), stream);
  if (e == hipSuccess && a.tokens > 0 && a.dx) e = run<true, false, kStore>(input_gradient(a), stream);
  if (e == hipSuccess && (a.dw_gate || a.dw_up || a.dw_down)) e = run<false, false, kStore>(weight_gradients(a), stream);
  return e;
}

}  // namespace knap
