// Differential attention, forward: per (sequence, head) of a packed bag
//   P_m = softmax(scale q_m k_m^T), O_m = P_m v (m = 1, 2),  out = O_1 - lambda O_2,
// where q_1, k_1 are the first d / 2 columns of a head's rows and q_2, k_2 the others.
//
// The structure is that of the forward of plain attention (knap_attn_fwd.hip): S_m^T = K_m Q_m^T with one query per lane, P_m^T as it
// comes out of that, packed, as the operand of O_m^T += V^T P_m^T, tiles of 64 keys through LDS, two buffers each.  Both maps are formed in
// one pass: the score products are as many as plain attention's (two halves of the columns), a fragment of V read from LDS feeds both
// maps' products, and nothing is formed twice.  6 L^2 d flops in all where four calls of plain attention (two maps, two halves of the values)
// would take 8.
//
// Row sums are taken over the probabilities as they are, in 32 bits, not over what is left of them in bf16: the log-sum is then as exact
// as its type allows.
#include "knap_diff.h"

namespace knap {

template <int D, bool CAUSAL>
__global__ __launch_bounds__(kThreads, 2) void diff_fwd_kernel(DiffFwdArgs a) {
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
  build_schedule<C::BM, kThreads, CAUSAL>(a.cu, a.n_seq, H, s_order, s_start, reinterpret_cast<int*>(&sK0[0]));
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float c = a.scale * kLog2e;
  const size_t row_stride = (size_t)H * D;
  const uint32_t row_bytes = (uint32_t)(row_stride * sizeof(__bf16));
  RowReader<D> k_rows;
  ColReader<D> v_cols;
  k_rows.init(lane);
  v_cols.init(lane);
  EvenQueue<0, 1> queue;
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
      const int q0 = q_tile * C::BM, q_row = q0 + 32 * wave + l32;
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
      load_tile(0, sK0, sV0);       // a barrier stands between the last reads of the buffers and this
      const uint32_t rows_bytes = (uint32_t)min(L - q0, C::BM) * row_bytes;
      const uint32_t off = (uint32_t)(32 * wave + l32) * row_bytes + (uint32_t)(16 * hh);
      bf16x8 qf[C::KC];
      {
        const auto rq = make_rsrc(a.q + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
        for (int cc = 0; cc < C::KC; ++cc) qf[cc] = __builtin_bit_cast(bf16x8, buffer_load16(rq, off + 32u * cc));
      }
      f32x16 o[2][C::DB];
      DiffSoftmax st[2];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int db = 0; db < C::DB; ++db) o[m][db] = zero16();
      wait_async_loads();
      lds_barrier();

      auto tile = [&](int t, const __bf16* tK, const __bf16* tV, __bf16* nK, __bf16* nV) {
        load_tile(t + 1, nK, nV);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int k0 = t * C::BN + 32 * half;
          if (k0 >= kv_end || (CAUSAL && k0 > q0 + 32 * wave + 31)) break;
          bf16x8 pb[2][2];
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            f32x16 s = zero16();
#pragma unroll
            for (int cc = 0; cc < C::KC / 2; ++cc) s = mfma32(k_rows.get(tK, 32 * half, m * C::KC / 2 + cc), qf[m * C::KC / 2 + cc], s);
            if (t >= first_masked) mask_half(s, kv_lim - k0, hh);
            st[m].template step<C::DB>(s, c, pb[m], o[m], hh);
          }
#pragma unroll
          for (int ck = 0; ck < 2; ++ck)
#pragma unroll
            for (int db = 0; db < C::DB; ++db) {
              const bf16x8 vt = v_cols.get(tV, 32 * half + 16 * ck, db);
              o[0][db] = mfma32(vt, pb[0][ck], o[0][db]);
              o[1][db] = mfma32(vt, pb[1][ck], o[1][db]);
            }
        }
        wait_async_loads();
        lds_barrier();
      };
      for (int t = 0; t < n_tiles; t += 2) {
        tile(t, sK0, sV0, sK1, sV1);
        if (t + 1 < n_tiles) tile(t + 1, sK1, sV1, sK0, sV0);
      }
      if (sub == 0 && queue.draws && tid == 0) next_ticket = atomicAdd(queue.ctr, 1u);

      float inv[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float l = st[m].l + xor32(st[m].l);
        inv[m] = 1.0f / l;
        const auto rl = make_rsrc(a.lse + ((size_t)m * H + head) * T + it.row0 + q0, (uint32_t)min(L - q0, C::BM) * 4u);
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, st[m].m_ref * a.scale + __logf(l)), rl,
                                              hh == 0 ? (32 * wave + l32) * 4 : 4 * C::BM, 0, 0);
      }
      const auto ro = make_rsrc(a.out + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
      for (int db = 0; db < C::DB; ++db) {
        f32x16 x;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = o[0][db][r] * inv[0] - lambda * (o[1][db][r] * inv[1]);
        store_block(ro, off + 64u * db, x, 1.0f);
      }
      if (a.out2) {
        const auto r2 = make_rsrc(a.out2 + seq_at + (size_t)q0 * row_stride, rows_bytes);
#pragma unroll
        for (int db = 0; db < C::DB; ++db) store_block(r2, off + 64u * db, o[1][db], inv[1]);
      }
    }
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
  hipLaunchKernelGGL(kernel, dim3(2 * cus), dim3(kThreads), dyn, stream, a);
  return hipGetLastError();
}

hipError_t launch_diff_fwd(const DiffFwdArgs& a, int d, bool causal, int cus, hipStream_t stream) {
  return d == 64 ? launch_diff_fwd_t<64>(a, causal, cus, stream) : launch_diff_fwd_t<128>(a, causal, cus, stream);
}

}  // namespace knap
