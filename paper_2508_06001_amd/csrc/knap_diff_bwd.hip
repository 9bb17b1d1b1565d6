// Differential attention, backward.  With P_m recomputed from q, k and the forward's log-sums, dP = dout v^T and D_m = sum_c dout_c O_m,c:
//   dS_1 = P_1 (dP - D_1),  dS_2 = -lambda P_2 (dP - D_2),  dq_m = scale dS_m k_m,  dk_m = scale dS_m^T q_m,
//   dv = (P_1 - lambda P_2)^T dout,  dlambda = - sum over rows of D_2.
// The products are as many as those of plain attention of the same d: the scores, dq and dk are two halves of the columns, dP and dv are
// one for both maps.  What is twice as much are the exponentials.  As there, dQ (by query tiles) and dK, dV (by key tiles) are kernels of
// their own that keep their sums in registers, and nothing is added up across workgroups but dlambda.
//
//   diff_dq_kernel      on the way in D_1 = sum dout out + lambda D_2 and D_2 = sum dout out2 of every row, from the rounded outputs, which is
//                       as exact as dS in bf16 can use, and the log-sums in base 2, both handed on in memory; dQ; and D_2 again in 32 bits,
//                       as sum_j P_2 dP, for dlambda (dout times the rounded out2 is off by 2^-9 a row, which a sum over rows of either
//                       sign does not average out against its own size)
//   diff_dkdv_kernel    dK, dV; behind its items dlambda, one workgroup a head, in a fixed order
// Probabilities are carried times 2^15 (the log-sums are stored that much smaller), which fp16 holds with 11 bits down to 2^-29: so
// that the waves that form dK get them from the waves that form dV with no rounding worth counting.  The results' factors take it out.
//
// What bounds them: vector arithmetic beside the matrix units (7.8 vector instructions a matrix one; these busy 42 % of the time in dQ, 51 % in
// dK/dV).  Measured at a settled clock (the first passes of a run take 5 to 20 % longer), dQ and dK/dV, us (TFLOP/s of their 6 and 8 L^2 d):
// 16384, 3 x 128, 710 (870) and 883 (930, on 192 of 256 CUs); 17 of 328 .. 4533 under the mask, 6 x 128, 250 (810) and 359 (750), 24 x 128, 1029 (790)
// and 1444 (750); 16384, 12 x 64, 1529 (810) and 3076 (540: a step's vector work is that of d = 128 for half the matrix work, at two waves a
// SIMD); 37 .. 311, 2 x 64, 14 and 17.
// No register is spilled in the loops over tiles: what the compiler puts aside (three values in the dK/dV kernel of four pairs, one in dQ at
// d = 128) it stores and reloads once an item, the ticket among it, or once a launch.
#include "knap_attn_dkdv.h"
#include "knap_attn_dq.h"
#include "knap_diff.h"

namespace knap {

constexpr float kDiffUp = 15.f;                       // log2 of what probabilities are carried times
constexpr float kDiffDown = 1.0f / 32768.f;

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// dQ: plain attention's structure.  S_m^T = K_m Q_m^T and dP^T = V dO^T put one query in each lane; dS_m^T is, unchanged, the operand of
// dQ_m^T += K_m^T dS_m^T with K^T read transposed from LDS.
template <int D, bool CAUSAL>
__global__ __launch_bounds__(kThreads, diff_workgroups(D)) void diff_dq_kernel(DiffBwdArgs a) {
  using C = DiffCfg<D>;
  extern __shared__ int s_dyn[];
  int* s_order = s_dyn;
  int* s_start = s_dyn + a.n_seq;
  __shared__ __attribute__((aligned(1024))) __bf16 sK0[C::TILE_ELEMS];
  __shared__ __attribute__((aligned(1024))) __bf16 sK1[C::TILE_ELEMS];
  __shared__ __attribute__((aligned(1024))) __bf16 sV0[C::TILE_ELEMS];
  __shared__ __attribute__((aligned(1024))) __bf16 sV1[C::TILE_ELEMS];
  __shared__ int s_ticket;
  static_assert(sizeof(__bf16) * C::TILE_ELEMS >= sizeof(int) * kThreads, "scan scratch must fit in a tile");

  const int T = a.cu[a.n_seq], H = a.H;
  const int n_items = build_schedule<C::BM, kThreads, false>(a.cu, a.n_seq, H, s_order, s_start, reinterpret_cast<int*>(&sK0[0]));
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float c = a.scale * kLog2e;
  const size_t row_stride = (size_t)H * D;
  const uint32_t row_bytes = (uint32_t)(row_stride * sizeof(__bf16));
  RowReader<D> rows;
  ColReader<D> cols;
  rows.init(lane);
  cols.init(lane);
  if (blockIdx.x == 0 && tid < 8) a.counters[tid] = 0u;      // of the launch behind this one
  StridedQueue queue;
  queue.init(a.dq_counters, n_items);
  int ticket = queue.first_ticket();
  while (ticket < queue.wide) {
    // under the mask the query tiles with most keys first, as in the forward (pairs in even shares, us: 17 of 328 .. 4533, 6 x 128, 320 -> 265; 4 of
    // 4096 235 -> 194; 32 of 200 33 -> 24; 8000, 12 x 64, 305 -> 239; 17 of 328 .. 4533, 24 x 128, 1038 -> 1045)
    WorkItem it;
    if constexpr (CAUSAL) it = decode_most_left<C::BM, true>(queue.item(ticket), a.cu, a.n_seq, H, s_order, s_start);
    else it = decode_tile_major<C::BM>(queue.item(ticket), a.cu, a.n_seq, H, s_order, s_start);
    const int L = it.len, head = __builtin_amdgcn_readfirstlane(it.head);
    const float lambda = a.lambda[head];
    unsigned next_ticket;      // thread 0 only
    const int q_tile = __builtin_amdgcn_readfirstlane(it.tile), q0 = q_tile * C::BM, q_row = q0 + 32 * wave + l32;
    const bool q_valid = q_row < L;
    const int kv_end = CAUSAL ? min(L, q0 + C::BM) : L;
    const int n_tiles = (kv_end + C::BN - 1) / C::BN;
    const int first_masked = CAUSAL ? 2 * q_tile : L / C::BN;
    const int kv_lim = CAUSAL ? q_row + 1 : L;
    const size_t seq_at = (size_t)it.row0 * row_stride + (size_t)head * D;
    auto load_tile = [&](int t, __bf16* dK, __bf16* dV) {
      const int kv0 = t * C::BN;
      const uint32_t bytes = (uint32_t)max(0, min(kv_end - kv0, C::BN)) * row_bytes;
      tile_load_async<D>(dK, make_rsrc(a.k + seq_at + (size_t)kv0 * row_stride, bytes), row_bytes, C::BN, wave, lane);
      tile_load_async<D>(dV, make_rsrc(a.v + seq_at + (size_t)kv0 * row_stride, bytes), row_bytes, C::BN, wave, lane);
    };
    const uint32_t rows_bytes = (uint32_t)min(L - q0, C::BM) * row_bytes;
    const uint32_t off = (uint32_t)(32 * wave + l32) * row_bytes + (uint32_t)(16 * hh);
    const size_t row_at = (size_t)head * T + it.row0 + (q_valid ? q_row : 0);
    const size_t second = (size_t)H * T;
    const float own_a = __builtin_fmaf(a.lse[row_at], kLog2e, -kDiffUp), own_b = __builtin_fmaf(a.lse[second + row_at], kLog2e, -kDiffUp);
    // +inf for rows past the end: P = 0
    const float lse_a = q_valid ? own_a : INFINITY, lse_b = q_valid ? own_b : INFINITY;
    // One tensor after the other (knap_attn_dq.h).  The lane holds half of its query's columns, its partner at lane ^ 32 the other half.
    bf16x8 qf[C::KC], dof[C::KC];
    float nd1, nd2;
    {
      const auto rq = make_rsrc(a.q + seq_at + (size_t)q0 * row_stride, rows_bytes);
      const auto rd = make_rsrc(a.dout + seq_at + (size_t)q0 * row_stride, rows_bytes);
      const auto ro = make_rsrc(a.out + seq_at + (size_t)q0 * row_stride, rows_bytes);
      const auto r2 = make_rsrc(a.out2 + seq_at + (size_t)q0 * row_stride, rows_bytes);
      bf16x8 of[C::KC], o2[C::KC];
#pragma unroll
      for (int cc = 0; cc < C::KC; ++cc) qf[cc] = __builtin_bit_cast(bf16x8, buffer_load16(rq, off + 32u * cc));
      KNAP_SCHED_FENCE();
#pragma unroll
      for (int cc = 0; cc < C::KC; ++cc) dof[cc] = __builtin_bit_cast(bf16x8, buffer_load16(rd, off + 32u * cc));
      KNAP_SCHED_FENCE();
#pragma unroll
      for (int cc = 0; cc < C::KC; ++cc) of[cc] = __builtin_bit_cast(bf16x8, buffer_load16(ro, off + 32u * cc));
      KNAP_SCHED_FENCE();
#pragma unroll
      for (int cc = 0; cc < C::KC; ++cc) o2[cc] = __builtin_bit_cast(bf16x8, buffer_load16(r2, off + 32u * cc));
      KNAP_SCHED_FENCE();
      load_tile(0, sK0, sV0);
      KNAP_SCHED_FENCE();
      const float d2_rounded = row_delta<D>(dof, o2);
      nd1 = -__builtin_fmaf(lambda, d2_rounded, row_delta<D>(dof, of));
      nd2 = -d2_rounded;
    }
    f32x16 acc[C::DB];
#pragma unroll
    for (int db = 0; db < C::DB; ++db) acc[db] = zero16();
    float d2 = 0.f;
    wait_async_loads();
    if (q_valid && hh == 0) {     // for the dK/dV kernel, behind the wait, which would wait for these stores as well
      a.nd1[row_at] = nd1;
      a.diff[row_at] = nd2 - nd1;
      a.lse_a[row_at] = own_a;
      a.lse_b[row_at] = own_b;
    }
    lds_barrier();

    // MASKED: a tile that crosses the sequence's end or the diagonal.  Keys that a query does not see score -inf: rows past the end
    // arrive as zeros, and exp2(-log-sum) of a score of zero may be infinite.  Halves that none of the wave's queries sees are left out.
    auto tile = [&](auto masked_tag, int t, const __bf16* tK, const __bf16* tV, __bf16* nK, __bf16* nV) __attribute__((always_inline)) {
      constexpr bool MASKED = decltype(masked_tag)::value;
      load_tile(t + 1, nK, nV);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int k0 = t * C::BN + 32 * half;
        if (MASKED && (k0 >= kv_end || (CAUSAL && k0 > q0 + 32 * wave + 31))) break;
        f32x16 dp = zero16();
#pragma unroll
        for (int cc = 0; cc < C::KC; ++cc) dp = mfma32(rows.get(tV, 32 * half, cc), dof[cc], dp);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          f32x16 s = zero16();
#pragma unroll
          for (int cc = 0; cc < C::KC / 2; ++cc) s = mfma32(rows.get(tK, 32 * half, m * C::KC / 2 + cc), qf[m * C::KC / 2 + cc], s);
          if constexpr (MASKED) mask_half(s, kv_lim - k0, hh);
          float ds[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float p = fast_exp2(__builtin_fmaf(s[r], c, -(m == 0 ? lse_a : lse_b)));
            if (m == 1) d2 = __builtin_fmaf(p, dp[r], d2);
            ds[r] = p * (dp[r] + (m == 0 ? nd1 : nd2));
          }
          const bf16x8 x0 = pack8(ds[0], ds[1], ds[2], ds[3], ds[4], ds[5], ds[6], ds[7]);
          const bf16x8 x1 = pack8(ds[8], ds[9], ds[10], ds[11], ds[12], ds[13], ds[14], ds[15]);
#pragma unroll
          for (int db = m * C::DB / 2; db < (m + 1) * C::DB / 2; ++db) {
            acc[db] = mfma32(cols.get(tK, 32 * half, db), x0, acc[db]);
            acc[db] = mfma32(cols.get(tK, 32 * half + 16, db), x1, acc[db]);
          }
        }
      }
      wait_async_loads();
      lds_barrier();
    };
    // (an even number of tiles in front of the masked ones under the mask, any otherwise)
    const int n_plain = min(n_tiles, first_masked);
    for (int t = 0; t < n_plain; t += 2) {
      tile(std::false_type{}, t, sK0, sV0, sK1, sV1);
      if (t + 1 < n_plain) tile(std::false_type{}, t + 1, sK1, sV1, sK0, sV0);
    }
    for (int t = n_plain; t < n_tiles; ++t) {
      const bool odd = t & 1;
      tile(std::true_type{}, t, odd ? sK1 : sK0, odd ? sV1 : sV0, odd ? sK0 : sK1, odd ? sV0 : sV1);
    }
    if (queue.draws && tid == 0) next_ticket = atomicAdd(queue.ctr, 1u);
    d2 += xor32(d2);
    if (q_valid && hh == 0) a.d2[row_at] = d2 * kDiffDown;
    const auto rg = make_rsrc(a.dq + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
    for (int db = 0; db < C::DB; ++db)
      store_block(rg, off + 64u * db, acc[db], db < C::DB / 2 ? a.scale * kDiffDown : -lambda * a.scale * kDiffDown);
    if (!queue.draws) return;
    if (tid == 0) s_ticket = drawn_ticket(queue, next_ticket);
    lds_barrier();
    ticket = __builtin_amdgcn_readfirstlane(s_ticket);
    lds_barrier();        // everyone has the ticket before the next one is put down
  }
}

// dK, dV: the structure of plain attention's kernel (knap_attn_dkdv.h), PAIRS pairs of waves, each pair with 64 keys of the tile and the
// two waves of a pair with a role each:
//   dV wave: keeps its K rows in registers; S_1, P_1, then S_2, P_2, both handed over as fp16 through LDS; dV += (P_1 - lambda P_2)^T dO;
//   dK wave: keeps its V rows in registers and runs one tile behind: dP - D_1 = dO V^T - D_1, dS_1 = P_1 (dP - D_1),
//            dS_2 = P_2 (dP - D_1 + (D_1 - D_2)), dK_m += dS_m^T Q_m; -lambda is taken in at the end.
// The dV wave's registers hold the scores of one map at a time: its P_1 comes back from the LDS that it was handed over through.
template <int D, int PAIRS>
struct DiffLane : DkdvLane<D, PAIRS> {
  using C = Bwd2Cfg<D, PAIRS>;
  static constexpr int P_BLOCK = 64 * 16, P_MAP = 2 * C::KB * P_BLOCK, P_TILE = 2 * P_MAP, P_PAIR = 2 * P_TILE;      // bytes
  __device__ __forceinline__ void init(int lane, int wave_, int role_, uint32_t row_bytes) {
    DkdvLane<D, PAIRS>::init(lane, wave_, role_, row_bytes);
    this->at.word = P_PAIR * this->pair + 16 * lane;
  }
};

// one slot of the ring: 32 rows of Q and dO, and 64 places each for their log-sums (two), -D_1 and D_1 - D_2 (wave w copies the w-th of them,
// the other waves nothing into the fifth)
struct DiffSlot {
  __bf16 *q, *dout;
  float* values;
};
constexpr int kDiffValues = 5 * 64;

// `draw` is called behind the last product, in front of the stores.
template <int D, int PAIRS, bool CAUSAL, class Draw>
__device__ __forceinline__ void diff_dkdv_tile(const DiffBwdArgs& g, const DiffSlot& r0, const DiffSlot& r1, const DiffSlot& r2, char* sP, char* sPark,
                                               const DiffLane<D, PAIRS>& me, const WorkItem& it, int head, int kv_tile, int T, Draw draw) {
  using C = Bwd2Cfg<D, PAIRS>;
  using W = DiffLane<D, PAIRS>;
  constexpr int KH = C::KC / 2, NH = C::NB / 2;
  const int L = it.len, role = me.role, pair = me.pair, wave = me.wave;
  const float c = g.scale * kLog2e, lambda = g.lambda[head];
  const size_t row_stride = (size_t)g.H * D;
  const uint32_t row_bytes = (uint32_t)(row_stride * sizeof(__bf16));
  const int kv0 = kv_tile * C::BN;
  const int q_first = CAUSAL ? kv0 : 0;       // queries this key tile meets: rows q_first .. L - 1; tiles and rows below count from it
  const int Lq = L - q_first;
  const size_t q_at = (size_t)(it.row0 + q_first) * row_stride + (size_t)head * D;
  const float* values = (wave == 0 ? g.lse_a : wave == 1 ? g.lse_b : wave == 2 ? g.nd1 : g.diff) + (size_t)head * T + it.row0 + q_first;
  const uint32_t value_bytes = wave < 4 ? 4u : 0u;
  const int n_tiles = (Lq + C::BM - 1) / C::BM;

  // PARKED: the last 16 columns lie in LDS, for which there is no register: spilled, their reloads would wait for the tile copies issued in
  // front of them (vector memory completes in issue order)
  constexpr int PARKED = D == 128 ? 1 : 0, KEPT = C::KC - PARKED;
  bf16x8 kvf[C::KB][KEPT];
  auto parked = [&](int kb, int w) { return reinterpret_cast<bf16x8*>(sPark + 1024 * (2 * wave + kb) + (LaneWord::lane4(w) << 2)); };
  {
    const auto r = make_rsrc((role == 0 ? g.k : g.v) + (size_t)(it.row0 + kv0) * row_stride + (size_t)head * D,
                             (uint32_t)min(L - kv0, C::BN) * row_bytes);
    const int w = me.at.fresh();
#pragma unroll
    for (int kb = 0; kb < C::KB; ++kb) {
      const uint32_t off = (uint32_t)(64 * pair + 32 * kb + LaneWord::l32(w)) * row_bytes + (uint32_t)LaneWord::hh16(w);
#pragma unroll
      for (int cc = 0; cc < KEPT; ++cc) kvf[kb][cc] = __builtin_bit_cast(bf16x8, buffer_load16(r, off + 32u * cc));
      if constexpr (PARKED) *parked(kb, w) = __builtin_bit_cast(bf16x8, buffer_load16(r, off + 32u * KEPT));
    }
  }
  f32x16 acc[C::KB][C::NB];
#pragma unroll
  for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
    for (int nb = 0; nb < C::NB; ++nb) acc[kb][nb] = zero16();

  // CAUSAL: step t works on query tile n_tiles - 1 - t, from the sequence's last one down to the diagonal
  auto issue_tile = [&](int t, const DiffSlot& to) {
    int q0, n_rows;
    if constexpr (CAUSAL) {
      q0 = max(0, n_tiles - 1 - t) * C::BM;
      n_rows = t < n_tiles ? min(Lq - q0, C::BM) : 0;
    } else {
      q0 = t * C::BM;
      n_rows = max(0, min(L - q0, C::BM));
    }
    const auto rq = make_rsrc(g.q + q_at + (size_t)q0 * row_stride, (uint32_t)n_rows * row_bytes);
    const auto rd = make_rsrc(g.dout + q_at + (size_t)q0 * row_stride, (uint32_t)n_rows * row_bytes);
#pragma unroll
    for (int r = 0; r < C::BM; r += 2 * PAIRS * W::ROWS_PER_INSTR) {
      uint32_t off = me.cp_off;
      if (r) asm volatile("" : "+v"(off));
      off += (uint32_t)r * row_bytes;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (__attribute__((address_space(3))) void*)(to.q + (me.cp_row0 + r) * Tile<D>::LD), 16, (int)off, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rd, (__attribute__((address_space(3))) void*)(to.dout + (me.cp_row0 + r) * Tile<D>::LD), 16, (int)off, 0, 0, 0);
    }
    __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(values + q0, (uint32_t)n_rows * value_bytes),
                                             (__attribute__((address_space(3))) void*)(to.values + 64 * min(wave, 4)), 4,
                                             LaneWord::lane4(me.at.fresh()), 0, 0, 0);
  };
  auto step_sync = [&]() {
    wait_async_loads();
    lds_barrier();
  };
  constexpr int AHEAD = 2;
  // x[kb] += tile rows (A, from LDS) x this wave's K or V rows, columns 16 FROM .. 16 TO
  auto first_product = [&](auto from_tag, auto to_tag, const __bf16* tA, int rb, int w, f32x16 (&x)[C::KB]) {
    constexpr int FROM = decltype(from_tag)::value, TO = decltype(to_tag)::value;
    bf16x8 af[C::KC], last[C::KB];
#pragma unroll
    for (int cc = FROM; cc < FROM + AHEAD && cc < TO; ++cc) af[cc] = me.rows.get(tA, rb, cc);
    KNAP_SCHED_FENCE();
#pragma unroll
    for (int cc = FROM; cc < TO; ++cc) {
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb) x[kb] = mfma32(af[cc], cc < KEPT ? kvf[kb][cc < KEPT ? cc : 0] : last[kb], x[kb]);
      if (cc + AHEAD < TO) af[cc + AHEAD] = me.rows.get(tA, rb, cc + AHEAD);
      if (cc + AHEAD == KEPT && cc + AHEAD < TO) {
#pragma unroll
        for (int kb = 0; kb < C::KB; ++kb) last[kb] = *parked(kb, w);
      }
      KNAP_SCHED_FENCE();
    }
  };
  // acc[kb][nb] += op[kb] x tile columns over the 16 queries of chunk cq, column blocks FROM .. TO
  auto second_product = [&](auto from_tag, auto to_tag, const __bf16* tB, int cb, int cq, const bf16x8 (&op)[C::KB]) {
    constexpr int FROM = decltype(from_tag)::value, TO = decltype(to_tag)::value;
    bf16x8 bf[C::NB];
#pragma unroll
    for (int nb = FROM; nb < FROM + 2 && nb < TO; ++nb) bf[nb] = me.cols.get(tB, cb, 16 * cq, nb);
    KNAP_SCHED_FENCE();
#pragma unroll
    for (int nb = FROM; nb < TO; ++nb) {
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb) acc[kb][nb] = mfma32(bf[nb], op[kb], acc[kb][nb]);
      if (nb + 2 < TO) bf[nb + 2] = me.cols.get(tB, cb, 16 * cq, nb + 2);
      KNAP_SCHED_FENCE();
    }
  };
  constexpr std::integral_constant<int, 0> n0{};
  constexpr std::integral_constant<int, KH> kh{};
  constexpr std::integral_constant<int, C::KC> kc{};
  constexpr std::integral_constant<int, NH> nh{};
  constexpr std::integral_constant<int, C::NB> nb_all{};
  // 16 bytes of this lane in block `b` of its pair's P of map m, tile t
  auto p_at = [&](int w, int t, int m, int b) {
    return reinterpret_cast<f16x8*>(sP + W::P_MAP * m + W::P_BLOCK * b + (w + (t & 1) * W::P_TILE));
  };
  auto dv_step = [&](int t, const DiffSlot& at) {
    const int rb = me.rows.fresh(), cb = me.cols.fresh(), w = me.at.fresh();
    // P_m of chunk cq and key block kb: register e of half h is query 8 (2 cq + h) + 4 hh + e
    auto exps = [&](const f32x16& s, const float* lse, int cq, float (&p)[8]) {
      const char* row = reinterpret_cast<const char*>(lse + 16 * cq) + LaneWord::hh16(w);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 lq = *reinterpret_cast<const f32x4*>(row + 32 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) p[4 * h + e] = fast_exp2(__builtin_fmaf(s[8 * cq + 4 * h + e], c, -lq[e]));
      }
    };
    f32x16 s[C::KB];
    // scores of queries before this lane's key are -inf: in one branch, not one for each probability, and with what it compares formed in it (formed
    // once for both maps it costs eight spilled registers, reloaded in every step, us: 17 of 328 .. 4533, 24 x 128, 1588 and 1435)
    auto mask = [&]() __attribute__((always_inline)) {
      if constexpr (CAUSAL) {
        const int back = n_tiles - 1 - t;
        if (back < C::BN / C::BM) {
          const int lanes = me.at.fresh();
          const int first_seen = 64 * pair + LaneWord::l32(lanes) - back * C::BM - LaneWord::hh16(lanes) / 4;      // of key block 0, 32 later of key block 1
#pragma unroll
          for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kb][r] = 8 * (r >> 2) + (r & 3) - 32 * kb < first_seen ? -INFINITY : s[kb][r];
        }
      }
    };
#pragma unroll
    for (int kb = 0; kb < C::KB; ++kb) s[kb] = zero16();
    first_product(n0, kh, at.q, rb, w, s);
    mask();
#pragma unroll
    for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
      for (int cq = 0; cq < 2; ++cq) {
        float p[8];
        exps(s[kb], at.values, cq, p);
        f16x8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (_Float16)p[e];
        *p_at(w, t, 0, 2 * kb + cq) = x;
      }
#pragma unroll
    for (int kb = 0; kb < C::KB; ++kb) s[kb] = zero16();
    first_product(kh, kc, at.q, rb, w, s);
    mask();
#pragma unroll
    for (int cq = 0; cq < 2; ++cq) {
      bf16x8 pa[C::KB];
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb) {
        float p[8];
        exps(s[kb], at.values + 64, cq, p);
        const f16x8 one = *p_at(w, t, 0, 2 * kb + cq);
        f16x8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = (_Float16)p[e];
          pa[kb][e] = (__bf16)__builtin_fmaf(-lambda, p[e], (float)one[e]);
        }
        *p_at(w, t, 1, 2 * kb + cq) = x;
      }
      second_product(n0, nb_all, at.dout, cb, cq, pa);
    }
  };
  // (a product with an fp16 factor is one instruction as a fused one)
  auto dk_step = [&](int u, const DiffSlot& at) {
    const int rb = me.rows.fresh(), cb = me.cols.fresh(), w = me.at.fresh();
    f32x16 dp[C::KB];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(reinterpret_cast<const char*>(at.values + 128) + LaneWord::hh16(w) + 32 * j);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int kb = 0; kb < C::KB; ++kb) dp[kb][4 * j + e] = x[e];
    }
    first_product(n0, kc, at.dout, rb, w, dp);
#pragma unroll
    for (int cq = 0; cq < 2; ++cq) {
      bf16x8 da[C::KB];
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb) {
        const f16x8 p = *p_at(w, u, 0, 2 * kb + cq);
#pragma unroll
        for (int e = 0; e < 8; ++e) da[kb][e] = (__bf16)__builtin_fmaf((float)p[e], dp[kb][8 * cq + e], 0.f);
      }
      second_product(n0, nh, at.q, cb, cq, da);
      const char* row = reinterpret_cast<const char*>(at.values + 192 + 16 * cq) + LaneWord::hh16(w);
      const f32x4 e0 = *reinterpret_cast<const f32x4*>(row), e1 = *reinterpret_cast<const f32x4*>(row + 32);
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb) {
        const f16x8 p = *p_at(w, u, 1, 2 * kb + cq);
#pragma unroll
        for (int e = 0; e < 8; ++e) da[kb][e] = (__bf16)__builtin_fmaf((float)p[e], dp[kb][8 * cq + e] + (e < 4 ? e0[e & 3] : e1[e & 3]), 0.f);
      }
      second_product(nh, nb_all, at.q, cb, cq, da);
    }
  };
  const int n_own = 64 * pair >= L - kv0 ? 0 : CAUSAL ? n_tiles - 2 * pair : n_tiles;      // see knap_attn_dkdv.h
#define KNAP_STEP(ROLE, t, cur, prev, nxt)                            \
  do {                                                                \
    issue_tile((t) + 1, r##nxt);                                      \
    if constexpr (ROLE == 0) {                                        \
      if ((t) < n_own) dv_step((t), r##cur);                          \
    } else {                                                          \
      if ((t) >= 1 && (t) <= n_own) dk_step((t) - 1, r##prev);        \
    }                                                                 \
    step_sync();                                                      \
  } while (0)
#define KNAP_ROLE_LOOP(ROLE)                                          \
  do {                                                                \
    int t = 0;                                                        \
    for (; t + 2 <= n_tiles; t += 3) {                                \
      KNAP_STEP(ROLE, t, 0, 2, 1);                                    \
      KNAP_STEP(ROLE, t + 1, 1, 0, 2);                                \
      KNAP_STEP(ROLE, t + 2, 2, 1, 0);                                \
    }                                                                 \
    if (t <= n_tiles) {                                               \
      KNAP_STEP(ROLE, t, 0, 2, 1);                                    \
      if (t + 1 <= n_tiles) KNAP_STEP(ROLE, t + 1, 1, 0, 2);          \
    }                                                                 \
  } while (0)
  issue_tile(0, r0);
  step_sync();
  if (role == 0) KNAP_ROLE_LOOP(0);
  else KNAP_ROLE_LOOP(1);
#undef KNAP_ROLE_LOOP
#undef KNAP_STEP
  draw();

  const auto rg = make_rsrc((role == 0 ? g.dv : g.dk) + (size_t)(it.row0 + kv0) * row_stride + (size_t)head * D,
                            (uint32_t)min(L - kv0, C::BN) * row_bytes);
  const int w_out = me.at.fresh();
#pragma unroll
  for (int kb = 0; kb < C::KB; ++kb) {
    const uint32_t off = (uint32_t)(64 * pair + 32 * kb + LaneWord::l32(w_out)) * row_bytes + (uint32_t)LaneWord::hh16(w_out);
#pragma unroll
    for (int nb = 0; nb < C::NB; ++nb)
      store_block(rg, off + 64u * nb, acc[kb][nb], kDiffDown * (role == 0 ? 1.0f : nb < NH ? g.scale : -lambda * g.scale));
  }
}

// dlambda of a head: minus the sum of its rows' D_2, by one workgroup
template <int THREADS>
__device__ __forceinline__ void diff_lambda(const DiffBwdArgs& a, int head, int T, float* s_sum) {
  const float* row = a.d2 + (size_t)head * T;
  float sum = 0.f;
#pragma unroll 8
  for (int t = threadIdx.x; t < T; t += THREADS) sum += row[t];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.f;
    for (int w = 0; w < THREADS / 64; ++w) sum += s_sum[w];
    a.dlambda[head] = -sum;
  }
  __syncthreads();
}

template <int D, int PAIRS, bool CAUSAL>
__global__ __launch_bounds__(128 * PAIRS, 2) void diff_dkdv_kernel(DiffBwdArgs a) {
  using C = Bwd2Cfg<D, PAIRS>;
  extern __shared__ int s_dyn[];
  int* s_order = s_dyn;
  int* s_start = s_dyn + a.n_seq;
#define KNAP_RING(i)                                                                    \
  __shared__ __attribute__((aligned(1024))) __bf16 sQ##i[C::TILE_ELEMS];                \
  __shared__ __attribute__((aligned(1024))) __bf16 sdO##i[C::TILE_ELEMS];               \
  __shared__ __attribute__((aligned(256))) float sValues##i[kDiffValues];
  KNAP_RING(0) KNAP_RING(1) KNAP_RING(2)
#undef KNAP_RING
  __shared__ __attribute__((aligned(1024))) char sP[PAIRS * DiffLane<D, PAIRS>::P_PAIR];
  __shared__ __attribute__((aligned(1024))) char sPark[D == 128 ? 2 * PAIRS * 2048 : 16];
  __shared__ int s_ticket;

  const int T = a.cu[a.n_seq];
  const int n_items = build_schedule<C::BN, C::THREADS, false>(a.cu, a.n_seq, a.H, s_order, s_start, reinterpret_cast<int*>(&sP[0]));
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the two waves of a pair sit on one SIMD where there are four pairs; at two pairs the second half of the grid swaps roles
  const int role = (wave / PAIRS) ^ (PAIRS == 2 ? (int)(blockIdx.x * 2 / gridDim.x) & 1 : 0);
  DiffLane<D, PAIRS> me;
  me.init(lane, wave, role, (uint32_t)((size_t)a.H * D * sizeof(__bf16)));
  const DiffSlot r0 = {sQ0, sdO0, sValues0}, r1 = {sQ1, sdO1, sValues1}, r2 = {sQ2, sdO2, sValues2};
  StridedQueue queue;
  queue.init(a.counters, n_items);
  for (int ticket = queue.first_ticket(); ticket < queue.wide;) {
    // longest items first: by what is left of the sequence under the mask (tile by tile of one sequence after the other, us: 4 of 4096, 6 x 128,
    // 383 -> 325; 32 of 450, 12 x 128, 155 -> 142; 17 of 328 .. 4533, 12 x 64, 542 -> 522), by sequence without it
    const int w = queue.item(ticket);
    const WorkItem it = CAUSAL ? decode_most_left<C::BN, false>(w, a.cu, a.n_seq, a.H, s_order, s_start)
                               : decode_tile_major<C::BN>(w, a.cu, a.n_seq, a.H, s_order, s_start);
    unsigned next_ticket;      // thread 0 only
    diff_dkdv_tile<D, PAIRS, CAUSAL>(a, r0, r1, r2, sP, sPark, me, it, it.head, it.tile, T, [&] {
      if (tid == 0 && queue.draws) next_ticket = atomicAdd(queue.ctr, 1u);
    });
    if (!queue.draws) break;
    if (tid == 0) s_ticket = queue.later_ticket(next_ticket);
    lds_barrier();
    ticket = __builtin_amdgcn_readfirstlane(s_ticket);
    lds_barrier();        // everyone has the ticket before the next one is put down
  }
  // dlambda by the workgroups from the last one on, which have the cheapest items or none
  __syncthreads();
  for (int head = (int)(gridDim.x - 1 - blockIdx.x); head < a.H; head += (int)gridDim.x) diff_lambda<C::THREADS>(a, head, T, reinterpret_cast<float*>(&sP[0]));
}

template <int D, int PAIRS, bool CAUSAL>
static hipError_t launch_diff_dkdv_t(const DiffBwdArgs& a, int grid, hipStream_t stream) {
  const size_t dyn = (size_t)(2 * a.n_seq + 1) * sizeof(int);
  hipLaunchKernelGGL((diff_dkdv_kernel<D, PAIRS, CAUSAL>), dim3(grid), dim3(128 * PAIRS), dyn, stream, a);
  return hipGetLastError();
}

template <int D, bool CAUSAL>
static hipError_t launch_diff_bwd_t(const DiffBwdArgs& a, int tokens, int cus, hipStream_t stream) {
  const size_t dyn = (size_t)(2 * a.n_seq + 1) * sizeof(int);
  hipLaunchKernelGGL((diff_dq_kernel<D, CAUSAL>), dim3(diff_workgroups(D) * cus), dim3(kThreads), dyn, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if constexpr (D == 64) return launch_diff_dkdv_t<64, 2, CAUSAL>(a, 2 * cus, stream);
  // d = 128: four pairs, 256 keys, fill a CU; two, 128 keys, leave half of its SIMDs' time unused (a step takes 0.86 of the time), but spread
  // few items over twice as many CUs.  Without the mask as long as each finds one of its own, us at four pairs and at two: one sequence of
  // 2000, 12 x 128, 131 and 108; of 5000, 6 x 128, 309 and 266; of 1000, 24 x 128, 75 and 60; 200, 150 and 90, 24 x 128, 24 and 19.
  // Under the mask, where items are half as long in the mean and the longest decide, up to two rounds of them, but for short sequences, whose
  // 256 keys are few items anyway: 16384, 3 x 128, 1018 and 883; 8000, 6 x 128, 510 and 445; 4 of 1000, 12 x 128, 86 and 72; 6 of
  // 768, 12 x 128, 71 and 67; 7 of 640 63 and 59; but 9 of 512 54 and 57; 12 of 300 41 and 45; 20 of 256 40 and 47.  The mean does not show a
  // long one among many short ones: 3000 and 20 of 100 take four, 209, where two would take 176.
  const double most = CAUSAL && tokens > 600 * (int64_t)a.n_seq ? 2.0 : 1.0;
  if (rounds(tokens, a.n_seq, a.H, 128, cus) <= most) return launch_diff_dkdv_t<128, 2, CAUSAL>(a, cus, stream);
  return launch_diff_dkdv_t<128, 4, CAUSAL>(a, cus, stream);
}

hipError_t launch_diff_bwd(const DiffBwdArgs& a, int d, bool causal, int tokens, int cus, hipStream_t stream) {
  if (d == 64) return causal ? launch_diff_bwd_t<64, true>(a, tokens, cus, stream) : launch_diff_bwd_t<64, false>(a, tokens, cus, stream);
  return causal ? launch_diff_bwd_t<128, true>(a, tokens, cus, stream) : launch_diff_bwd_t<128, false>(a, tokens, cus, stream);
}

}  // namespace knap
