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
// 7.4 vector instructions a matrix one, the matrix units busy 57 % of the time.  Measured at a settled clock (the first passes of a run take
// 5 to 20 % longer), us (TFLOP/s): 4173 and 4096, 24 x 128, 622 (1010); 17 of 328 .. 4533 under the mask, 6 x 128, 219 (920), 24 x 128, 876 (920);
// 16384, 3 x 128, 653 (950, on the 75 % of the workgroups that have an item); 16384, 12 x 64, 1309 (940); 37 .. 311, 2 x 64, 11.
// Under the mask items are single query tiles, those with most keys first, drawn one by one (pairs of a long and a short tile in even shares, as
// plain attention has them, us: 17 of 328 .. 4533, 6 x 128, 255 -> 231; 4 of 4096 200 -> 170; 32 of 200, 6 x 128, 28 -> 19; 8000, 12 x 64, 260 -> 203;
// the longest items alone decide for 16384, 3 x 128, 433 -> 473).  Parts of 64 queries for few items, as plain attention has them, cost more
// than they gain here: one of 2000, 12 x 128, 73 in parts and 66; of 1000, 24 x 128, 43 and 39.
// With probabilities in bf16 out is off by 2.5e-3 in the 2-norm where its own rounding alone is 1.7e-3: they are the operand of a matrix
// product with v, whose type they take.
//
// Row sums are taken over the probabilities as they are, in 32 bits, not over what is left of them in bf16: the log-sum is then as exact
// as its type allows.
#include "knap_diff.h"

namespace knap {

// The keys go through in halves of 32.  A stage is a half and a map; three stages that follow each other are in work at a time, in one slot of
// the pipeline: the scores of the last one, the probabilities of the middle one, the product with the values of the first one.  No
// product of a slot waits for its arithmetic, nor the other way round; the stage whose sums a moving reference rescales is of the other
// map than the one whose products run.  K runs half a tile ahead of V: a turn (two slots, one barrier) reads the keys of half h + 1 and
// the values of half h, while the keys of h + 2 and the values of h + 1 are copied.
// Workgroups a CU, two and three at d = 64, us: 16384, 12 heads, 1635 and 1393; 10 of 310 .. 6795, 48 heads, 2009 and 1906; 17 of 328 .. 4533, 12 heads, under
// the mask, 302 and 269 (8000, 12 heads, 201 and 210: its longest items alone decide).
template <int D, bool CAUSAL>
__global__ __launch_bounds__(kThreads, diff_workgroups(D)) void diff_fwd_kernel(DiffFwdArgs a) {
  using C = DiffCfg<D>;
  constexpr int KH = C::KC / 2, DB = C::DB, ROWS = 32, TILE = ROWS * Tile<D>::LD;
  extern __shared__ int s_dyn[];
  int* s_order = s_dyn;
  int* s_start = s_dyn + a.n_seq;
  __shared__ __attribute__((aligned(1024))) __bf16 sK0[TILE];
  __shared__ __attribute__((aligned(1024))) __bf16 sK1[TILE];
  __shared__ __attribute__((aligned(1024))) __bf16 sV0[TILE];
  __shared__ __attribute__((aligned(1024))) __bf16 sV1[TILE];
  // The last columns of each map's q, KH - KEPT chunks of 16, lie in LDS: there are no registers for them, and spilled, their reloads in
  // every turn would wait for the copies in front of them (4173 and 4096, 24 x 128, us: 702 -> 662; 32 of 450 234 -> 184)
  constexpr int KEPT = D == 128 ? KH - (CAUSAL ? 2 : 1) : KH;
  __shared__ __attribute__((aligned(1024))) char sPark[KEPT < KH ? 2 * (KH - KEPT) * 4096 : 16];
  __shared__ int s_ticket;
  static_assert(sizeof(__bf16) * TILE >= sizeof(int) * kThreads, "scan scratch must fit in a tile");

  const int T = a.cu[a.n_seq], H = a.H;
  const int n_items = build_schedule<C::BM, kThreads, false>(a.cu, a.n_seq, H, s_order, s_start, reinterpret_cast<int*>(&sK0[0]));
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // what follows from the lane is formed where it is used, from this one register: the loop has none to spare
  auto here = [&]() __attribute__((always_inline)) { int x = lane; asm volatile("" : "+v"(x)); return x; };
  const float c = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, a.scale * kLog2e)));      // (a scalar register)
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
  StridedQueue queue;
  queue.init(a.counters, n_items);
  int ticket = queue.first_ticket();
  while (ticket < queue.wide) {
    WorkItem it;
    if constexpr (CAUSAL) it = decode_most_left<C::BM, true>(queue.item(ticket), a.cu, a.n_seq, H, s_order, s_start);
    else it = decode_tile_major<C::BM>(queue.item(ticket), a.cu, a.n_seq, H, s_order, s_start);
    const int L = it.len, head = __builtin_amdgcn_readfirstlane(it.head);
    const float lambda = a.lambda[head];
    unsigned next_ticket;      // thread 0 only
    const int q0 = __builtin_amdgcn_readfirstlane(it.tile) * C::BM;
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
    bf16x8 qf[2][KEPT];
    auto parked = [&](int m, int i) { return reinterpret_cast<bf16x8*>(sPark + 4096 * (m * (KH - KEPT) + i - KEPT) + 1024 * wave + 16 * here()); };
    {
      const int ln = here();
      const uint32_t off = (uint32_t)(32 * wave + (ln & 31)) * row_bytes + (uint32_t)(16 * (ln >> 5));
      const auto rq = make_rsrc(a.q + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
#pragma unroll
        for (int i = 0; i < KEPT; ++i) qf[m][i] = __builtin_bit_cast(bf16x8, buffer_load16(rq, off + 32u * (m * KH + i)));
#pragma unroll
        for (int i = KEPT; i < KH; ++i) *parked(m, i) = __builtin_bit_cast(bf16x8, buffer_load16(rq, off + 32u * (m * KH + i)));
      }
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
        bf16x8 last[KH];
#pragma unroll
        for (int i = 0; i < KH; ++i) {
          sn = mfma32(ak[i], i < KEPT ? qf[NEXT][i < KEPT ? i : 0] : last[i], i == 0 ? zero16() : sn);
          if (i + 2 >= KEPT && i + 2 < KH) last[i + 2] = *parked(NEXT, i + 2);
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
        for (int i = 0; i < KH; ++i) s0 = mfma32(ak[i], i < KEPT ? qf[0][i < KEPT ? i : 0] : *parked(0, i), i == 0 ? zero16() : s0);
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
    if (queue.draws && tid == 0) next_ticket = atomicAdd(queue.ctr, 1u);

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
    if (!queue.draws) return;
    if (tid == 0) s_ticket = drawn_ticket(queue, next_ticket);
    lds_barrier();
    ticket = __builtin_amdgcn_readfirstlane(s_ticket);
    lds_barrier();        // everyone has the ticket before the next one is put down
  }
}

template <int D>
static hipError_t launch_diff_fwd_t(const DiffFwdArgs& a, bool causal, int cus, hipStream_t stream) {
  const size_t dyn = (size_t)(2 * a.n_seq + 1) * sizeof(int);
  auto* kernel = causal ? diff_fwd_kernel<D, true> : diff_fwd_kernel<D, false>;
  hipLaunchKernelGGL(kernel, dim3(diff_workgroups(D) * cus), dim3(kThreads), dyn, stream, a);
  return hipGetLastError();
}

hipError_t launch_diff_fwd(const DiffFwdArgs& a, int d, bool causal, int cus, hipStream_t stream) {
  return d == 64 ? launch_diff_fwd_t<64>(a, causal, cus, stream) : launch_diff_fwd_t<128>(a, causal, cus, stream);
}

}  // namespace knap
