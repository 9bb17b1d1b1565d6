// Gated feed-forward block, forward, of few tokens (the next ones of some sequences, at most 32): both products of knap_ffn.hip where the weights' bytes are all
// that counts.  Every weight is read once, straight into registers; x, h and the sums stay in the caches.
//   v_mfma_f32_16x16x32_bf16   A: lane holds row lane % 16, k's 8 (lane / 16) .. + 7, B: column lane % 16, the same k's,
//                              D: registers r are rows 4 (lane / 16) + r of column lane % 16
// A workgroup forms 16 results (rows of the weights) of all tokens, 16 tokens a block of columns; its waves share the k's in runs of 32 STEPS, so that a row's
// bytes are asked for in whole lines, with the next run's loads under way, and add up their sums in LDS in a fixed order.
// Bound by HBM; what more tokens add is x and h, which every workgroup reads from L2.  Waves and steps as measured on weights that are in no cache, us (the
// second product behind the +; 4 waves of 2 steps and 8 of 4 as they are here, against 8 and 16 waves of 4): one token 2048 x 5504 12.9 + 8.2 (15.2 + 8.7),
// 4096 x 10944 35.6 + 15.0 (36.1 + 15.8; 5.0 and 6.0 TB/s); 24 tokens 47.5 + 29.2 (52.1 + 30.2).  32 rows of the weights a workgroup read x half as often, but
// are fewer workgroups: 24 tokens 60 + 47.
#include "knap_device.h"
#include "knap_kernels.h"

namespace knap {

struct FewArgs {
  const __bf16 *w0, *w1, *x;      // rows of K; w1: of the second product of a pair
  int64_t x_stride;
  int tokens, N, K;
  __bf16 *out, *gate, *up;        // out: h or y; gate, up: of a pair, or nullptr
  int64_t out_stride;
  bool gelu;
};

// as in knap_ffn.hip
__device__ __forceinline__ float gated(float a, float b, bool gelu) {
  float u = a;
  if (gelu) {
    const float c = __builtin_fminf(__builtin_fmaxf(a, -16.f), 16.f);
    u = 1.5957691216057308f * __builtin_fmaf(0.044715f * c, c * c, c);
  }
  return a * __builtin_amdgcn_rcpf(1.f + fast_exp2(-kLog2e * u)) * b;
}

template <int BLOCKS, bool PAIR, int WAVES, int STEPS>
__global__ __launch_bounds__(64 * WAVES) void ffn_few_kernel(FewArgs a) {
  constexpr int MATS = PAIR ? 2 : 1, RUN = 32 * STEPS;
  constexpr int kNowhere = 0x7fffffe0;      // a byte offset behind every descriptor
  __shared__ f32x4 s_sum[WAVES][MATS * BLOCKS][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = (int)blockIdx.x * 16, row = lane & 15, part = 8 * (lane >> 4);
  const uint32_t w_bytes = (uint32_t)min(16, a.N - n0) * (uint32_t)a.K * 2u;
  const __amdgpu_buffer_rsrc_t r0 = make_rsrc(a.w0 + (int64_t)n0 * a.K, w_bytes), r1 = make_rsrc((PAIR ? a.w1 : a.w0) + (int64_t)n0 * a.K, w_bytes);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x, (uint32_t)(((int64_t)(a.tokens - 1) * a.x_stride + a.K) * 2));
  const int w_row = row * a.K * 2, x_row = row * (int)a.x_stride * 2, x_block = 32 * (int)a.x_stride;
  u32x4 w[2][MATS][STEPS], x[2][BLOCKS][STEPS];
  auto load = [&](int k0, int set) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int k = k0 + 32 * s + part;
      const bool there = k < a.K;      // K is a multiple of 8: whole units
      w[set][0][s] = buffer_load16(r0, there ? w_row + 2 * k : kNowhere);
      if constexpr (PAIR) w[set][1][s] = buffer_load16(r1, there ? w_row + 2 * k : kNowhere);
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) x[set][b][s] = buffer_load16(rx, there ? x_row + b * x_block + 2 * k : kNowhere);
    }
  };
  f32x4 acc[MATS][BLOCKS];
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) acc[m][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](int set) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int m = 0; m < MATS; ++m)
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
          acc[m][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[set][m][s]), __builtin_bit_cast(bf16x8, x[set][b][s]),
                                                              acc[m][b], 0, 0, 0);
  };
  int k = wave * RUN;
  load(k, 0);      // zeros behind K
  while (true) {
    load(k + WAVES * RUN, 1);
    multiply(0);
    k += WAVES * RUN;
    if (k >= a.K) break;
    load(k + WAVES * RUN, 0);
    multiply(1);
    k += WAVES * RUN;
    if (k >= a.K) break;
  }
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) s_sum[wave][m * BLOCKS + b][lane] = acc[m][b];
  __syncthreads();
  if (wave >= BLOCKS) return;
  const int token = 16 * wave + row, n = n0 + 4 * (lane >> 4);
  f32x4 sum[MATS];
#pragma unroll
  for (int m = 0; m < MATS; ++m) {
    sum[m] = s_sum[0][m * BLOCKS + wave][lane];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) sum[m] += s_sum[v][m * BLOCKS + wave][lane];
  }
  if (token >= a.tokens || n >= a.N) return;
  auto store = [&](__bf16* p, const f32x4& v) {
    *reinterpret_cast<bf16x4*>(p) = pack4(v[0], v[1], v[2], v[3]);
  };
  __bf16* out = a.out + token * a.out_stride + n;
  if constexpr (PAIR) {
    f32x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = gated(sum[0][e], sum[1][e], a.gelu);
    store(out, h);
    if (a.gate) {
      store(a.gate + (int64_t)token * a.N + n, sum[0]);
      store(a.up + (int64_t)token * a.N + n, sum[1]);
    }
  } else {
    store(out, sum[0]);
  }
}

template <bool PAIR, int WAVES, int STEPS>
static hipError_t launch_few(const FewArgs& a, hipStream_t stream) {
  const dim3 grid((a.N + 15) / 16), block(64 * WAVES);
  if (a.tokens <= 16) hipLaunchKernelGGL((ffn_few_kernel<1, PAIR, WAVES, STEPS>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((ffn_few_kernel<2, PAIR, WAVES, STEPS>), grid, block, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_ffn_few(const FfnArgs& f, hipStream_t stream) {
  FewArgs a{};
  a.w0 = f.w_gate; a.w1 = f.w_up; a.x = f.x; a.x_stride = f.x_stride;
  a.tokens = f.tokens; a.N = f.hidden; a.K = f.width;
  a.out = f.h; a.out_stride = f.hidden; a.gate = f.gate; a.up = f.up;
  a.gelu = f.gelu;
  const hipError_t e = launch_few<true, 4, 2>(a, stream);
  if (e != hipSuccess) return e;
  a.w0 = f.w_down; a.w1 = nullptr; a.x = f.h; a.x_stride = f.hidden;
  a.N = f.width; a.K = f.hidden;
  a.out = f.y; a.out_stride = f.y_stride; a.gate = a.up = nullptr;
  return launch_few<false, 8, 4>(a, stream);
}

}  // namespace knap
