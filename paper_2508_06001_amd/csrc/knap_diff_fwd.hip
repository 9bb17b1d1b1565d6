// Differential attention, forward: per (sequence, head) of a packed bag
//   P_m = softmax(scale q_m k_m^T), O_m = P_m v (m = 1, 2),  out = O_1 - lambda O_2,
// where q_1, k_1 are the first d / 2 columns of a head's rows and q_2, k_2 the others.
//
// The structure is that of the forward of plain attention (knap_attn_fwd.hip): S_m^T = K_m Q_m^T with one query per lane, P_m^T as it
// comes out of that, packed, as the operand of O_m^T += V^T P_m^T, the keys through LDS, two buffers each.  Both maps are formed in
// one pass: the score products are as many as plain attention's (two halves of the columns), and nothing is formed twice: 6 L^2 d flops
// in all, where four calls of plain attention (two maps, two halves of the values) would take 8.
//
// What bounds it: two exponentials a score pair where plain attention has one, beside 24 matrix instructions a half of 32 keys and wave;
// the vector unit has 1.5 times plain attention's work a product.  Measured, us (credited TFLOP/s): 2 x 4292 and 37 .. 384, 24 x 128, 655
// (960); 12 x 64 under the mask, tiny 10.6; 8192 x 2 and 16384, 3 x 128, 716 (770 of them on the 75 % of the workgroups that have an item).
// With probabilities in bf16 out is off by 2.5e-3 in the 2-norm where its own rounding alone is 1.7e-3: they are the operand of a matrix
// product with v, whose type they take.
//
// Row sums are taken over the probabilities as they are, in 32 bits, not over what is left of them in bf16: the log-sum is then as exact
// as its type allows.
#include "knap_diff.h"

namespace knap {

// 64 query rows of a sequence and head, from q0 on: waves w and w + 2 share 32 of them, one taking the first 32 keys of every 64, the other the
// second; the two halves of each softmax are merged through LDS at the end.  A barrier has to stand between this and whatever reads or
// fills the tiles before or behind it.
struct DiffTiles {
  __bf16 *k[4], *v[4];      // 32 rows each; two pairs in turn
};

template <int D, bool CAUSAL>
__device__ __forceinline__ void diff_fwd_part(const DiffFwdArgs& a, const DiffTiles& lds, const WorkItem& it, int head, int q0, int T, int lane, int wave) {
  using C = DiffCfg<D>;
  constexpr int KH = C::KC / 2, DB = C::DB, ROWS = 32;
  const int L = it.len, l32 = lane & 31, hh = lane >> 5;
  const int rb = __builtin_amdgcn_readfirstlane(wave & 1), kh = __builtin_amdgcn_readfirstlane(wave >> 1);
  const float c = a.scale * kLog2e, lambda = a.lambda[head];
  const size_t row_stride = (size_t)a.H * D;
  const uint32_t row_bytes = (uint32_t)(row_stride * sizeof(__bf16));
  const int kv_end = CAUSAL ? min(L, q0 + 64) : L, n_tiles = (kv_end + 63) / 64;
  const size_t seq_at = (size_t)it.row0 * row_stride + (size_t)head * D;
  auto copy = [&](const __bf16* src, int kv0, __bf16* dst) {
    tile_load_async<D>(dst, make_rsrc(src + seq_at + (size_t)kv0 * row_stride, (uint32_t)max(0, min(kv_end - kv0, ROWS)) * row_bytes), row_bytes, ROWS,
                       wave, lane);
  };
  RowReaderX<D> k_rows;
  ColReaderX<D> v_cols;
  k_rows.init(lane);
  v_cols.init(lane);
  const uint32_t rows_bytes = (uint32_t)min(L - q0, 64) * row_bytes;
  const uint32_t off = (uint32_t)(32 * rb + l32) * row_bytes + (uint32_t)(16 * hh);
  bf16x8 qf[C::KC];
  const auto rq = make_rsrc(a.q + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
  for (int cc = 0; cc < C::KC; ++cc) qf[cc] = __builtin_bit_cast(bf16x8, buffer_load16(rq, off + 32u * cc));
  f32x16 o[2][DB];
  DiffSoftmax st[2];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int db = 0; db < DB; ++db) o[m][db] = zero16();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    copy(a.k, 32 * i, lds.k[i]);
    copy(a.v, 32 * i, lds.v[i]);
  }
  wait_async_loads();
  lds_barrier();
  const int kv_lim = CAUSAL ? q0 + 32 * rb + l32 + 1 : L, all_see = CAUSAL ? q0 + 32 * rb + 1 : L, none_see = CAUSAL ? q0 + 32 * rb + 32 : L;
  auto tile = [&](int t, const __bf16* tK, const __bf16* tV, __bf16* nK0, __bf16* nK1, __bf16* nV0, __bf16* nV1) __attribute__((always_inline)) {
    copy(a.k, 64 * t + 64, nK0);
    copy(a.k, 64 * t + 96, nK1);
    copy(a.v, 64 * t + 64, nV0);
    copy(a.v, 64 * t + 96, nV1);
    const int k0 = 64 * t + 32 * kh;
    if (k0 < min(none_see, kv_end)) {
      const int kb = k_rows.fresh(), vb = v_cols.fresh();
      bf16x8 pb[2][2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        f32x16 s = zero16();
#pragma unroll
        for (int cc = 0; cc < KH; ++cc) s = mfma32(k_rows.get(tK, kb, m * KH + cc), qf[m * KH + cc], s);
        if (k0 + ROWS > all_see) mask_half(s, kv_lim - k0, hh);
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = fast_exp2(__builtin_fmaf(s[r], c, -st[m].mc));
          sum += p;
          pb[m][r >> 3][r & 7] = (__bf16)p;
        }
        st[m].template settle<DB>(s, c, sum, pb[m], o[m]);
      }
#pragma unroll
      for (int j = 0; j < 2 * DB; ++j) {
        const bf16x8 vt = v_cols.get(tV, vb, 16 * (j / DB), j % DB);
#pragma unroll
        for (int m = 0; m < 2; ++m) o[m][j % DB] = mfma32(vt, pb[m][j / DB], o[m][j % DB]);
      }
    }
    wait_async_loads();
    lds_barrier();
  };
  for (int t = 0; t < n_tiles; t += 2) {
    tile(t, kh == 0 ? lds.k[0] : lds.k[1], kh == 0 ? lds.v[0] : lds.v[1], lds.k[2], lds.k[3], lds.v[2], lds.v[3]);
    if (t + 1 < n_tiles) tile(t + 1, kh == 0 ? lds.k[2] : lds.k[3], kh == 0 ? lds.v[2] : lds.v[3], lds.k[0], lds.k[1], lds.v[0], lds.v[1]);
  }

  // merge, a map at a time: the waves of the second keys put down reference, sum and output, those of the first take them up
  constexpr int PER = DB / 2;       // blocks of 32 columns that a buffer of 32 rows holds in 32 bits
  float* part_ml = reinterpret_cast<float*>(lds.k[0]) + 128 * rb;
  auto part_o = [&](int db) { return reinterpret_cast<float*>(rb == 0 ? lds.k[2 + db / PER] : lds.v[2 + db / PER]) + 1024 * (db % PER); };
  float inv[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    if (kh == 1) {
      part_ml[lane] = st[m].m_ref;
      part_ml[64 + lane] = st[m].l;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 x = {o[m][db][4 * j], o[m][db][4 * j + 1], o[m][db][4 * j + 2], o[m][db][4 * j + 3]};
          *reinterpret_cast<f32x4*>(part_o(db) + (64 * j + lane) * 4) = x;
        }
    }
    lds_barrier();
    if (kh == 0) {
      const float m_ref = st[m].m_ref, m_other = part_ml[lane], l_other = part_ml[64 + lane];
      const float m_new = fmaxf(m_ref, m_other);
      const float a_own = m_new == m_ref ? 1.f : fast_exp2((m_ref - m_new) * c), a_other = m_new == m_other ? 1.f : fast_exp2((m_other - m_new) * c);
      const float l_half = st[m].l * a_own + l_other * a_other, l = l_half + xor32(l_half);
      inv[m] = 1.0f / l;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(part_o(db) + (64 * j + lane) * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[m][db][4 * j + e] = o[m][db][4 * j + e] * a_own + x[e] * a_other;
        }
      const auto rl = make_rsrc(a.lse + ((size_t)m * a.H + head) * T + it.row0 + q0, (uint32_t)min(L - q0, 64) * 4u);
      __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, m_new * a.scale + __logf(l)), rl, hh == 0 ? (32 * rb + l32) * 4 : 4 * 64, 0, 0);
    }
    lds_barrier();
  }
  if (kh == 0) {
    const auto ro = make_rsrc(a.out + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      f32x16 x;
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = o[0][db][r] * inv[0] - lambda * (o[1][db][r] * inv[1]);
      store_block(ro, off + 64u * db, x, 1.0f);
    }
    if (a.out2) {
      const auto r2 = make_rsrc(a.out2 + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
      for (int db = 0; db < DB; ++db) store_block(r2, off + 64u * db, o[1][db], inv[1]);
    }
  }
}

// The keys go through in halves of 32.  A stage is a half and a map; three stages that follow each other are in work at a time, in one slot of
// the pipeline: the scores of the last one, the probabilities of the middle one, the product with the values of the first one.  No
// product of a slot waits for its arithmetic, nor the other way round; the stage whose sums a moving reference rescales is of the other
// map than the one whose products run.  K runs half a tile ahead of V: a turn (two slots, one barrier) reads the keys of half h + 1 and
// the values of half h, while the keys of h + 2 and the values of h + 1 are copied.
template <int D, bool CAUSAL>
__global__ __launch_bounds__(kThreads, 2) void diff_fwd_kernel(DiffFwdArgs a) {
  using C = DiffCfg<D>;
  constexpr int KH = C::KC / 2, DB = C::DB, ROWS = 32, TILE = ROWS * Tile<D>::LD;
  extern __shared__ int s_dyn[];
  int* s_order = s_dyn;
  int* s_start = s_dyn + a.n_seq;
  __shared__ __attribute__((aligned(1024))) __bf16 sK0[TILE];
  __shared__ __attribute__((aligned(1024))) __bf16 sK1[TILE];
  __shared__ __attribute__((aligned(1024))) __bf16 sV0[TILE];
  __shared__ __attribute__((aligned(1024))) __bf16 sV1[TILE];
  __shared__ __attribute__((aligned(1024))) __bf16 sK2[TILE], sK3[TILE], sV2[TILE], sV3[TILE];      // of the parts alone
  __shared__ int s_ticket;
  static_assert(sizeof(__bf16) * TILE >= sizeof(int) * kThreads, "scan scratch must fit in a tile");

  const int T = a.cu[a.n_seq], H = a.H;
  build_schedule<C::BM, kThreads, CAUSAL>(a.cu, a.n_seq, H, s_order, s_start, reinterpret_cast<int*>(&sK0[0]));
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // what follows from the lane is formed where it is used, from this one register: the loop has none to spare
  auto here = [&]() __attribute__((always_inline)) { int x = lane; asm volatile("" : "+v"(x)); return x; };
  const float c = a.scale * kLog2e;
  const size_t row_stride = (size_t)H * D;
  const uint32_t row_bytes = (uint32_t)(row_stride * sizeof(__bf16));
  RowReaderX<D> k_rows;
  ColReaderX<D> v_cols;
  k_rows.init(lane);
  v_cols.init(lane);
  // where this lane's 16 bytes of a copied half lie in the tensor: a wave's instruction copies CP_ROWS rows, the waves and then the
  // instructions in turn; the swizzle looks at a row's low four bits alone, which a second instruction has in common
  constexpr int CP_ROWS = 512 / D;
  static_assert(4 * CP_ROWS % 16 == 0 && ROWS % (4 * CP_ROWS) == 0, "");
  const int cp_row = wave * CP_ROWS + lane / Tile<D>::CPR;
  const uint32_t cp_off = (uint32_t)cp_row * row_bytes + (uint32_t)Tile<D>::chunk_pos(cp_row, lane % Tile<D>::CPR) * 16u;
  constexpr int SPLIT = CAUSAL ? 4 : 2;     // narrow items (64 queries) of a wide one
  EvenQueue<SPLIT, 1> queue;
  queue.init(a.counters);
  if (tid < 64) even_shares(queue, a.n_seq, s_start, lane);
  __syncthreads();
  deal_even<C::BM, CAUSAL>(queue, a.cu, a.n_seq, s_order, s_start);

  int ticket = queue.first_ticket();
  while (ticket < queue.wide) {
    const WorkItem it = decode_even<C::BM, CAUSAL>(ticket, queue, a.cu, a.n_seq, H, s_order, s_start);
    const int L = it.len, head = __builtin_amdgcn_readfirstlane(it.head);
    const int other = (L + C::BM - 1) / C::BM - 1 - it.tile;     // CAUSAL: the pair of query tiles {other, tile}, the long one first
    const float lambda = a.lambda[head];
    unsigned next_ticket;      // thread 0 only
    for (int sub = 0; sub < (CAUSAL && it.tile != other ? 2 : 1); ++sub) {
      const int q_tile = __builtin_amdgcn_readfirstlane(!CAUSAL ? it.tile : sub == 0 ? other : it.tile);
      const int q0 = q_tile * C::BM;
      const int kv_end = CAUSAL ? min(L, q0 + C::BM) : L;
      const int n_half = (kv_end + ROWS - 1) / ROWS;
      // halves that this wave's queries see, none where its rows lie past the end: it then only copies; the last one is masked under the
      // mask (its diagonal) and where the sequence ends in it
      const int n_own = q0 + 32 * wave >= L ? 0 : CAUSAL ? min(n_half, q0 / ROWS + wave + 1) : n_half;
      const size_t seq_at = (size_t)it.row0 * row_stride + (size_t)head * D;
      auto copy = [&](const __bf16* src, int h, __bf16* dst) __attribute__((always_inline)) {
        const int kv0 = h * ROWS;
        const auto r = make_rsrc(src + seq_at + (size_t)kv0 * row_stride, (uint32_t)max(0, min(kv_end - kv0, ROWS)) * row_bytes);
#pragma unroll
        for (int i = 0; i < ROWS / (4 * CP_ROWS); ++i) {
          uint32_t o = cp_off;
          if (i) asm volatile("" : "+v"(o));     // formed here, not kept in a register of its own through the loop
          __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(dst + (4 * i + wave) * CP_ROWS * Tile<D>::LD), 16,
                                                   (int)(o + (uint32_t)(4 * i * CP_ROWS) * row_bytes), 0, 0, 0);
        }
      };
      copy(a.k, 0, sK0);       // a barrier stands between the last reads of the buffers and this
      const uint32_t rows_bytes = (uint32_t)min(L - q0, C::BM) * row_bytes;
      bf16x8 qf[C::KC];
      {
        const int ln = here();
        const uint32_t off = (uint32_t)(32 * wave + (ln & 31)) * row_bytes + (uint32_t)(16 * (ln >> 5));
        const auto rq = make_rsrc(a.q + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
        for (int cc = 0; cc < C::KC; ++cc) qf[cc] = __builtin_bit_cast(bf16x8, buffer_load16(rq, off + 32u * cc));
      }
      f32x16 o[2][DB];
      DiffSoftmax st[2];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int db = 0; db < DB; ++db) o[m][db] = zero16();
      wait_async_loads();
      lds_barrier();
      copy(a.v, 0, sV0);
      copy(a.k, 1, sK1);

      bf16x8 ak[KH];
      auto keys = [&](const __bf16* tK, int kb, int m, int i) __attribute__((always_inline)) { ak[i] = k_rows.get(tK, kb, m * KH + i); };
      // One slot: the scores sn of map NEXT (QK: its keys in `ak`), the probabilities pn of scores s against map NOW's reference (PR), the
      // product of map NEXT's probabilities pb with the values tV (PV).  Groups of a product each, fences between them, so that the order
      // below is the order issued; `behind(i)` goes into the groups of the second product.
      auto slot = [&](auto qk_tag, auto pr_tag, auto pv_tag, auto next_tag, const f32x16& s, f32x16& sn, const bf16x8 (&pb)[2], bf16x8 (&pn)[2],
                      const __bf16* tV, int vb, float& sum, auto behind) __attribute__((always_inline)) {
        constexpr bool QK = decltype(qk_tag)::value, PR = decltype(pr_tag)::value, PV = decltype(pv_tag)::value;
        constexpr int NEXT = decltype(next_tag)::value, NOW = 1 - NEXT;
        constexpr int GROUPS = (QK ? KH : 0) + (PV ? 2 * DB : 0), PER = PR ? (16 + GROUPS - 1) / GROUPS : 0;
        const float mc = st[NOW].mc;
        float p[16];
        int r = 0;
        auto form = [&]() __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < PER; ++e) {
            if (r < 16) {
              p[r] = fast_exp2(__builtin_fmaf(s[r], c, -mc));
              sum += p[r];
              pn[r >> 3][r & 7] = (__bf16)p[r];
            }
            ++r;
          }
        };
        bf16x8 vt[2 * DB];
        auto value = [&](int j) __attribute__((always_inline)) { vt[j] = v_cols.get(tV, vb, 16 * (j / DB), j % DB); };
        sum = 0.f;
        if constexpr (PV && !QK) { value(0); value(1); KNAP_SCHED_FENCE(); }
        if constexpr (QK) {
#pragma unroll
          for (int i = 0; i < KH; ++i) {
            sn = mfma32(ak[i], qf[NEXT * KH + i], i == 0 ? zero16() : sn);
            if (PV && i >= KH - 2) value(i - (KH - 2));
            form();
            KNAP_SCHED_FENCE();
          }
        }
        if constexpr (PV) {
#pragma unroll
          for (int j = 0; j < 2 * DB; ++j) {
            o[NEXT][j % DB] = mfma32(vt[j], pb[j / DB], o[NEXT][j % DB]);
            if (j + 2 < 2 * DB) value(j + 2);
            behind(j);
            form();
            KNAP_SCHED_FENCE();
          }
        }
      };
      constexpr std::true_type yes{};
      constexpr std::false_type no{};
      constexpr std::integral_constant<int, 0> map0{};
      constexpr std::integral_constant<int, 1> map1{};
      f32x16 s0, s1;            // scores of the maps
      bf16x8 pb0[2], pb1[2];    // their probabilities
      auto nothing = [](int) {};
      const bool masked = CAUSAL || (n_own == n_half && kv_end % ROWS != 0);
      auto mask = [&](f32x16& s, int h) __attribute__((always_inline)) {
        if (masked && h == n_own - 1) {
          const int ln = here();
          mask_half(s, (CAUSAL ? q0 + 32 * wave + (ln & 31) + 1 : L) - h * ROWS, ln >> 5);
        }
        KNAP_SCHED_FENCE();
      };
      if (n_own > 0) {
        float sum;
        {
          const int kb = k_rows.fresh();
#pragma unroll
          for (int i = 0; i < KH; ++i) keys(sK0, kb, 0, i);
#pragma unroll
          for (int i = 0; i < KH; ++i) s0 = mfma32(ak[i], qf[i], i == 0 ? zero16() : s0);
#pragma unroll
          for (int i = 0; i < KH; ++i) keys(sK0, kb, 1, i);
        }
        mask(s0, 0);
        slot(yes, yes, no, map1, s0, s1, pb1, pb0, sV0, 0, sum, nothing);
        st[0].template settle<DB>(s0, c, sum, pb0, o[0]);
        mask(s1, 0);
      }
      // the second map of half h and the first of half h + 1 go through the softmax
      auto turn = [&](int h, const __bf16* tK, const __bf16* tV, __bf16* nK, __bf16* nV) __attribute__((always_inline)) {
        wait_async_loads();
        lds_barrier();
        const int kb = k_rows.fresh(), vb = v_cols.fresh();
#pragma unroll
        for (int i = 0; i < KH; ++i) keys(tK, kb, 0, i);
        copy(a.k, h + 2, nK);
        copy(a.v, h + 1, nV);
        float sum;
        slot(yes, yes, yes, map0, s1, s0, pb0, pb1, tV, vb, sum, [&](int j) __attribute__((always_inline)) { if (j >= 2 * DB - KH) keys(tK, kb, 1, j - (2 * DB - KH)); });
        st[1].template settle<DB>(s1, c, sum, pb1, o[1]);
        mask(s0, h + 1);
        slot(yes, yes, yes, map1, s0, s1, pb1, pb0, tV, vb, sum, nothing);
        st[0].template settle<DB>(s0, c, sum, pb0, o[0]);
        mask(s1, h + 1);
      };
      int h = 0;
      for (; h < n_own - 1; h += 2) {
        turn(h, sK1, sV0, sK0, sV1);
        if (h + 2 < n_own) turn(h + 1, sK0, sV1, sK1, sV0);
      }
      h = max(n_own - 1, 0);
      // the last half's second map, and its products; then, and for waves without rows from the start, the others' turns: copies alone
      wait_async_loads();
      lds_barrier();
      if (h + 1 < n_half) {
        copy(a.k, h + 2, (h & 1) ? sK1 : sK0);
        copy(a.v, h + 1, (h & 1) ? sV0 : sV1);
      }
      if (n_own > 0) {
        const __bf16* tV = (h & 1) ? sV1 : sV0;
        const int vb = v_cols.fresh();
        float sum;
        slot(no, yes, yes, map0, s1, s0, pb0, pb1, tV, vb, sum, nothing);
        st[1].template settle<DB>(s1, c, sum, pb1, o[1]);
        slot(no, no, yes, map1, s0, s1, pb1, pb0, tV, vb, sum, nothing);
      }
      for (++h; h < n_half; ++h) {
        wait_async_loads();
        lds_barrier();
        if (h + 1 < n_half) {
          copy(a.k, h + 2, (h & 1) ? sK1 : sK0);
          copy(a.v, h + 1, (h & 1) ? sV0 : sV1);
        }
      }
      if (sub == 0 && queue.draws && tid == 0) next_ticket = atomicAdd(queue.ctr, 1u);

      const int ln = here();
      const uint32_t off = (uint32_t)(32 * wave + (ln & 31)) * row_bytes + (uint32_t)(16 * (ln >> 5));
      float inv[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float l = st[m].l + xor32(st[m].l);
        inv[m] = 1.0f / l;
        const auto rl = make_rsrc(a.lse + ((size_t)m * H + head) * T + it.row0 + q0, (uint32_t)min(L - q0, C::BM) * 4u);
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, st[m].m_ref * a.scale + __logf(l)), rl,
                                              ln < 32 ? (32 * wave + ln) * 4 : 4 * C::BM, 0, 0);
      }
      const auto ro = make_rsrc(a.out + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        f32x16 x;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = o[0][db][r] * inv[0] - lambda * (o[1][db][r] * inv[1]);
        store_block(ro, off + 64u * db, x, 1.0f);
      }
      if (a.out2) {
        const auto r2 = make_rsrc(a.out2 + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
        for (int db = 0; db < DB; ++db) store_block(r2, off + 64u * db, o[1][db], inv[1]);
      }
      lds_barrier();        // nobody reads a tile any longer
    }
    if (!queue.draws) return;
    if (tid == 0) s_ticket = drawn_ticket(queue, next_ticket);
    lds_barrier();
    ticket = __builtin_amdgcn_readfirstlane(s_ticket);
    lds_barrier();        // everyone has the ticket before the next one is put down
  }
  // few items, or those of a thin last round: in parts of 64 queries (EvenQueue::deal)
  const DiffTiles tiles = {{sK0, sK1, sK2, sK3}, {sV0, sV1, sV2, sV3}};
  for (int part = ticket - queue.wide; part >= 0 && part < queue.parts;) {
    const WorkItem it = decode_even<C::BM, CAUSAL>(queue.item_of_part(part), queue, a.cu, a.n_seq, H, s_order, s_start);
    const int head = __builtin_amdgcn_readfirstlane(it.head), other = (it.len + C::BM - 1) / C::BM - 1 - it.tile, sub = (part % SPLIT) >> 1;
    const int q0 = __builtin_amdgcn_readfirstlane((CAUSAL && sub == 0 ? other : it.tile) * C::BM + 64 * (part & 1));
    if (q0 < it.len && !(CAUSAL && sub == 1 && it.tile == other)) diff_fwd_part<D, CAUSAL>(a, tiles, it, head, q0, T, lane, wave);
    if (!queue.draws) return;         // every part was a first ticket
    if (tid == 0) {
      const unsigned drawn = atomicAdd(queue.ctr, 1u);
      s_ticket = drawn_ticket(queue, drawn);
    }
    lds_barrier();                    // (and the tiles are no longer read)
    part = __builtin_amdgcn_readfirstlane(s_ticket) - queue.wide;
    lds_barrier();                    // everyone has the ticket before it is drawn again
  }
}

template <int D>
static hipError_t launch_diff_fwd_t(const DiffFwdArgs& a, bool causal, int cus, hipStream_t stream) {
  const size_t dyn = (size_t)(2 * a.n_seq + 1) * sizeof(int);
  auto* kernel = causal ? diff_fwd_kernel<D, true> : diff_fwd_kernel<D, false>;
  hipLaunchKernelGGL(kernel, dim3(2 * cus), dim3(kThreads), dyn, stream, a);
  return hipGetLastError();
}

hipError_t launch_diff_fwd(const DiffFwdArgs& a, int d, bool causal, int cus, hipStream_t stream) {
  return d == 64 ? launch_diff_fwd_t<64>(a, causal, cus, stream) : launch_diff_fwd_t<128>(a, causal, cus, stream);
}

}  // namespace knap
