// Residual norm, backward (forward: knap_residual_norm_fwd.hip), from dx' (the residual's own gradient) and dy:
//   g = dy (1 + scale) w,  X = dx' + rstd (g - [mean g] - xh mean(g xh)),  dx = X
//   e = alpha gate wp X,   df = rp (e - [mean e] - fh mean(e fh)), or e without a post norm;  [] for layer norm alone
// and, over the rows of a sequence, A = sum dy, B = sum dy xh, C = sum X fh:
//   dshift = A,  dscale = w B,  dgate = alpha wp C,  dw = sum over sequences of (1 + scale) B,  dwp = alpha sum of gate C.
// x' is formed again from x and f, as the forward had it before its rounding: the same bytes as x' itself would be.
// Bound by HBM: x, f, dx' and dy are read once, dx and df written once.  A, B and C of the sequence that a workgroup is in stay in its
// registers; at the sequence's end (or its own) they go to the workspace, row `workgroup + sequence` of them: both only ever rise along the
// rows, so that no two meet.  A second kernel adds up each sequence's rows in a fixed order: no atomics, the same bits every time.
// 31464 rows of 1536 in bf16, layer norm: 580 MB in 109 us (5.3 TB/s) and 5.6 for the sums; 24576 of 2048, x in 32 bits, RMS on both sides: 906 MB in 194
// (4.7) and 8.8; 7584 of 1003 in 32 bits, columns singly: 183 MB in 42 (4.3) and 7.5.  These are of one set of inputs, part of which stays in the last cache;
// of three in turn, in no cache, with the sums: 149 us, 241 and 64.
#include "knap_residual_norm.h"

#include <algorithm>

namespace knap {

template <class C, class TX, class TB, bool POST>
__global__ __launch_bounds__(C::THREADS, C::THREADS > 512 ? 4 : 2) void residual_norm_bwd_kernel(ResidualArgs a) {
  __shared__ float s_sum[2][2 * C::ROWS * C::THREADS / 64];
  __shared__ float s_cols[C::GROUPS > 1 ? C::THREADS * C::COLS : 1];
  constexpr bool AHEAD = residual_ahead<C, TX>();
  const int g = threadIdx.x % C::LANES, group = threadIdx.x / C::LANES;
  const int width = a.width;
  const float n = (float)width;
  const bool layer = a.norm == KNAP_NORM_LAYER, post_layer = a.post_norm == KNAP_NORM_LAYER;
  const TX* x_base = static_cast<const TX*>(a.x);
  const TB* f_base = static_cast<const TB*>(a.f);
  const TX* dxo_base = static_cast<const TX*>(a.dx_out);
  const TB* dy_base = static_cast<const TB*>(a.dy);
  TX* dx_base = static_cast<TX*>(a.dx);
  TB* df_base = static_cast<TB*>(a.df);
  RowCursor at;
  at.start(a, (int)min((int64_t)blockIdx.x * a.chunk, a.rows), (int)min((int64_t)(blockIdx.x + 1) * a.chunk, a.rows));
  RowRaw<C, TX> raw_x[C::ROWS], raw_dxo[C::ROWS];
  RowRaw<C, TB> raw_f[C::ROWS], raw_dy[C::ROWS];
  float raw_stats[C::ROWS][4];
  auto load = [&](const RowCursor& c) {
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      const int64_t first = (int64_t)c.row + k * C::GROUPS, row = first + group;
      load_row<C, TX>(RowPlace<C, TX>(x_base, a.x_stride, first, group, c.end, width), g, raw_x[k]);
      // nothing is read where there is no such tensor: a descriptor of no bytes, and zeros
      load_row<C, TX>(RowPlace<C, TX>(dxo_base, a.dx_out_stride, first, group, dxo_base ? c.end : 0, width), g, raw_dxo[k]);
      load_row<C, TB>(RowPlace<C, TB>(f_base, a.f_stride, first, group, f_base ? c.end : 0, width), g, raw_f[k]);
      load_row<C, TB>(RowPlace<C, TB>(dy_base, a.dy_stride, first, group, dy_base ? c.end : 0, width), g, raw_dy[k]);
      const bool there = row < c.end;
      raw_stats[k][0] = there && dy_base ? a.stats[row] : 0.f;
      raw_stats[k][1] = there && dy_base ? a.stats[a.rows + row] : 0.f;
      raw_stats[k][2] = there && POST ? a.stats[2 * a.rows + row] : 0.f;
      raw_stats[k][3] = POST ? (there ? a.stats[3 * a.rows + row] : 0.f) : 1.f;
    }
  };
  if (AHEAD && at.row < at.limit) load(at);
  int seq = -1, turn = 0;
  bool first_sum = true;
  float gz[C::COLS], sw[C::COLS], sa[C::COLS], sb[C::COLS], sc[C::COLS];
  // one column's sums of the sequence just left
  auto leave = [&](int c, float A, float B, float D) {
    float* mine = a.partial + ((int64_t)blockIdx.x + seq) * 3 * width + c;
    mine[0] = A;
    mine[width] = B;
    mine[2 * width] = D;
    if (!a.totals) return;
    auto mod = [&](const void* v, int64_t stride) {
      const int64_t i = (int64_t)seq * stride + c;
      return a.mod_bf16 ? (float)static_cast<const __bf16*>(v)[i] : static_cast<const float*>(v)[i];
    };
    const float tb = B * (a.scale ? 1.f + mod(a.scale, a.mod_stride) : 1.f);
    const float tc = D * a.alpha * (a.gate ? mod(a.gate, a.gate_stride) : 1.f);
    float* total = a.totals + (int64_t)blockIdx.x * 2 * width + c;
    total[0] = first_sum ? tb : total[0] + tb;
    total[width] = first_sum ? tc : total[width] + tc;
  };
  auto flush = [&](int g) {
    if (!a.partial) return;
    if constexpr (C::GROUPS == 1) {
#pragma unroll
      for (int i = 0; i < C::COLS; ++i)
        if (norm_has<C>(g, i, width)) leave(norm_col<C>(g, i), sa[i], sb[i], sc[i]);
    } else {
      // a thread's columns are the same at every turn, in registers and in the totals
      constexpr int OWN = C::COLS / C::GROUPS + 1;
      float mine[3][OWN];
#pragma unroll
      for (int v = 0; v < 3; ++v) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < C::COLS; ++i)
          if (norm_has<C>(g, i, width)) s_cols[group * width + norm_col<C>(g, i)] = v == 0 ? sa[i] : v == 1 ? sb[i] : sc[i];
        __syncthreads();
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
          const int c = threadIdx.x + o * C::THREADS;
          mine[v][o] = 0.f;
          if (c < width) {
#pragma unroll
            for (int k = 0; k < C::GROUPS; ++k) mine[v][o] += s_cols[k * width + c];
          }
        }
      }
#pragma unroll
      for (int o = 0; o < OWN; ++o) {
        const int c = threadIdx.x + o * C::THREADS;
        if (c < width) leave(c, mine[0][o], mine[1][o], mine[2][o]);
      }
    }
    first_sum = false;
  };
  while (true) {
    const bool done = at.row >= at.limit;
    if (done || at.seq != seq) {
      // what is done once a sequence forms its addresses here: outside of the loop they would take the registers of the rows
      int own = g;
      asm volatile("" : "+v"(own));
      if (seq >= 0) flush(own);
      if (done) return;
      seq = at.seq;
      load_gate<C>(a, seq, own, gz);
      load_scale<C>(a, seq, own, sw);
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) sa[i] = sb[i] = sc[i] = 0.f;
    }
    if (!AHEAD) load(at);
    // x' in place of x, the normed f
    float x[C::ROWS][C::COLS], f[C::ROWS][C::COLS], mean[C::ROWS], rstd[C::ROWS], rp[C::ROWS];
    RowRaw<C, TX> dxo[C::ROWS];
    RowRaw<C, TB> dy[C::ROWS];
    float sums[2 * C::ROWS];
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      mean[k] = raw_stats[k][0];
      rstd[k] = raw_stats[k][1];
      rp[k] = raw_stats[k][3];
      dxo[k] = raw_dxo[k];
      dy[k] = raw_dy[k];
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) {
        f[k][i] = POST ? (raw_f[k].get(i) - raw_stats[k][2]) * rp[k] : raw_f[k].get(i);
        // without a norm no gradient depends on x', whatever it holds: a zero by a product of it would be none of an infinity
        x[k][i] = dy_base ? __builtin_fmaf(f[k][i], gz[i], raw_x[k].get(i)) : 0.f;
      }
    }
    const RowCursor now = at;
    at.step(a, C::PASS);
    if (AHEAD && at.row < at.limit) load(at);
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) {
        x[k][i] = (x[k][i] - mean[k]) * rstd[k];      // xh from here on
        const float y = dy[k].get(i), gi = y * sw[i];
        sa[i] += y;
        sb[i] = __builtin_fmaf(y, x[k][i], sb[i]);
        s1 += gi;
        s2 = __builtin_fmaf(gi, x[k][i], s2);
      }
      sums[2 * k] = s1;
      sums[2 * k + 1] = s2;
    }
    if (dy_base) {
      row_sums<C>(sums, s_sum[turn]);
      turn ^= 1;
    }
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      const float m1 = layer ? sums[2 * k] / n : 0.f, m2 = sums[2 * k + 1] / n;
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) {
        const float X = __builtin_fmaf(rstd[k], __builtin_fmaf(dy[k].get(i), sw[i], -m1) - x[k][i] * m2, dxo[k].get(i));
        x[k][i] = X;                                  // X from here on
        sc[i] = __builtin_fmaf(X, f[k][i], sc[i]);
        if constexpr (POST) {
          const float e = X * gz[i];
          s1 += e;
          s2 = __builtin_fmaf(e, f[k][i], s2);
        }
      }
      sums[2 * k] = s1;
      sums[2 * k + 1] = s2;
      if (dx_base) store_row<C, TX>(RowPlace<C, TX>(dx_base, a.dx_stride, (int64_t)now.row + k * C::GROUPS, group, now.end, width), g, x[k]);
    }
    if (!df_base) continue;
    if constexpr (POST) {
      row_sums<C>(sums, s_sum[turn]);
      turn ^= 1;
    }
#pragma unroll
    for (int k = 0; k < C::ROWS; ++k) {
      const float m1 = post_layer ? sums[2 * k] / n : 0.f, m2 = sums[2 * k + 1] / n;
      float df[C::COLS];
#pragma unroll
      for (int i = 0; i < C::COLS; ++i) df[i] = POST ? rp[k] * (__builtin_fmaf(x[k][i], gz[i], -m1) - f[k][i] * m2) : x[k][i] * gz[i];
      store_row<C, TB>(RowPlace<C, TB>(df_base, a.df_stride, (int64_t)now.row + k * C::GROUPS, group, now.end, width), g, df);
    }
  }
}

// Adds up what the workgroups left.  blockIdx.y: a sequence, or n_seq for the sums over all of them; COLS columns of the three (two) sums
// for a workgroup of SLICES * COLS threads.
template <int COLS, int SLICES>
__global__ __launch_bounds__(COLS * SLICES) void residual_norm_sum_kernel(ResidualArgs a, int cols) {
  __shared__ float s_part[SLICES][COLS];
  const int c = threadIdx.x % COLS, slice = threadIdx.x / COLS;
  const int s = blockIdx.y, width = a.width;
  const bool whole = s == a.n_seq;
  const int j = (int)blockIdx.x * COLS + c;
  int64_t last = a.rows;
  if (a.cu) last = min(last, (int64_t)max(0, a.cu[a.n_seq]));
  int64_t r0 = 0, r1 = last;
  if (a.cu && !whole) {
    r0 = max(0, a.cu[s]);
    r1 = min(last, (int64_t)a.cu[s + 1]);
  }
  const int v = j / width, col = j - v * width;
  float* out = nullptr;
  if (j < cols) {
    if (whole) out = v == 0 ? a.dweight : v == 1 ? a.dpost_weight : nullptr;
    else out = v == 0 ? a.dshift : v == 1 ? a.dscale : a.dgate;
  }
  float sum = 0.f;
  if (out && r1 > r0) {
    const int g0 = whole ? 0 : (int)(r0 / a.chunk), g1 = (int)((r1 - 1) / a.chunk);
    const int64_t pitch = (whole ? 2 : 3) * (int64_t)width;
    const float* from = whole ? a.totals + j : a.partial + (int64_t)s * pitch + j;
#pragma unroll 8
    for (int i = g0 + slice; i <= g1; i += SLICES) sum += from[i * pitch];
  }
  s_part[slice][c] = sum;
  __syncthreads();
  if (slice != 0 || !out) return;
  sum = 0.f;
  for (int k = 0; k < SLICES; ++k) sum += s_part[k][c];
  auto weight = [&](const void* w) { return !w ? 1.f : a.w_bf16 ? (float)static_cast<const __bf16*>(w)[col] : static_cast<const float*>(w)[col]; };
  if (whole) out[col] = sum;
  else if (v == 0) out[(int64_t)s * a.dmod_stride + col] = sum;
  else if (v == 1) out[(int64_t)s * a.dmod_stride + col] = weight(a.weight) * sum;
  else out[(int64_t)s * a.dgate_stride + col] = a.alpha * weight(a.post_weight) * sum;
}

static hipError_t launch_sums(const ResidualArgs& a, int groups, hipStream_t stream) {
  // columns of the three sums of a sequence, or of the two over all of them, that anyone wants
  const bool each = a.dshift || a.dscale || a.dgate, whole = a.dweight || a.dpost_weight;
  if ((!each || a.n_seq == 0) && !whole) return hipSuccess;
  const int cols = 3 * a.width;
  const dim3 grid((cols + 63) / 64, a.n_seq + (whole ? 1 : 0));
  // a sequence's rows of sums are `groups` / n_seq on the average: threads side by side accordingly
  if (groups > 32 * a.n_seq) hipLaunchKernelGGL((residual_norm_sum_kernel<64, 16>), grid, dim3(1024), 0, stream, a, cols);
  else hipLaunchKernelGGL((residual_norm_sum_kernel<64, 4>), grid, dim3(256), 0, stream, a, cols);
  return hipGetLastError();
}

template <class TX, class TB, bool WIDE>
static hipError_t launch_bwd_t(ResidualArgs a, int cus, hipStream_t stream) {
  return residual_form<WIDE>(a.width, [&](auto cfg) {
    using C = decltype(cfg);
    // workgroups a CU: more leave more sums to add up (31464 rows of 1536 in 16 bits, two and three a CU: 132 and 140 us), which rows of 32 bits
    // make up for (24576 of 2048: 225 and 209; 7584 of 1003: 56 and 50)
    a.chunk = residual_chunk(a.rows, std::min((sizeof(TX) == 4 ? 3 : 2) * cus, kResidualMaxGroups), C::PASS);
    const int groups = (int)((a.rows + a.chunk - 1) / a.chunk);
    if (groups > 0) {
      hipLaunchKernelGGL((a.post_norm == KNAP_NORM_NONE ? residual_norm_bwd_kernel<C, TX, TB, false> : residual_norm_bwd_kernel<C, TX, TB, true>), dim3(groups), dim3(C::THREADS), 0, stream, a);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return launch_sums(a, groups, stream);
  });
}

hipError_t launch_residual_norm_bwd(const ResidualArgs& a, bool x_bf16, bool b_bf16, bool wide, int cus, hipStream_t stream) {
  if (x_bf16) return wide ? launch_bwd_t<__bf16, __bf16, true>(a, cus, stream) : launch_bwd_t<__bf16, __bf16, false>(a, cus, stream);
  if (b_bf16) return wide ? launch_bwd_t<float, __bf16, true>(a, cus, stream) : launch_bwd_t<float, __bf16, false>(a, cus, stream);
  return wide ? launch_bwd_t<float, float, true>(a, cus, stream) : launch_bwd_t<float, float, false>(a, cus, stream);
}

}  // namespace knap
