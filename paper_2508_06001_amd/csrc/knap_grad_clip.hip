// Global norm of many gradients and clipping by it:
//   S = sum g^2 over all tensors,  c = min(1, max_norm / (sqrt(S) + eps)),  out = c g.
// Bound by HBM: every gradient is read once for S and once more for the product, which is written once.  Workgroups take chunks of a plan
// in turn, whose records say where they lie.  Squares and sums are in 64 bits (of which the card does as many as of 32): no gradient that is finite
// overflows or vanishes in them, and the norm is right to its last bit in 32.  Every workgroup leaves one sum, which a second launch adds up in a fixed order.
// The second pass goes through the plan from its end: what the first has read last is in the caches still, and stays there, since the second reads and writes
// past them.  339.8 million elements in bf16 (2.04 GB moved), us: both passes from the front 381, the stores past the caches 364, from the end 357, the
// loads past them as well 327 (6.2 TB/s; 110 and 211 the two passes); 34.7 million, most in 32 bits: 67.6, 55.9, 55.5, 55.0.
#include "knap_device.h"
#include "knap_kernels.h"

#include <algorithm>

namespace knap {

constexpr int kGradThreads = 256;

// 16 bytes as floats
template <class T> struct Unit;
template <> struct Unit<__bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void open(u32x4 x, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __builtin_bit_cast(float, x[e] << 16);
      v[2 * e + 1] = __builtin_bit_cast(float, x[e] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 close(const float (&v)[8]) {
    return __builtin_bit_cast(u32x4, pack8(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]));
  }
};
template <> struct Unit<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void open(u32x4 x, float (&v)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_bit_cast(float, (uint32_t)x[e]);
  }
  static __device__ __forceinline__ u32x4 close(const float (&v)[4]) {
    u32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __builtin_bit_cast(uint32_t, v[e]);
    return x;
  }
};

// A chunk: `count` elements of T from p + start.  Where p lies on 16 bytes every chunk does.
template <class T>
__device__ __forceinline__ double chunk_squares(const T* p, int count) {
  using U = Unit<T>;
  constexpr int TURNS = KNAP_GRAD_CHUNK / (U::N * kGradThreads);
  double s0 = 0.0, s1 = 0.0;
  if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, (uint32_t)count / U::N * 16u);
    u32x4 x[TURNS];
#pragma unroll
    for (int i = 0; i < TURNS; ++i) x[i] = buffer_load16(r, (threadIdx.x + i * kGradThreads) * 16u);      // zeros behind the chunk
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      float v[U::N];
      U::open(x[i], v);
#pragma unroll
      for (int e = 0; e < U::N; e += 2) {
        s0 = __builtin_fma((double)v[e], (double)v[e], s0);
        s1 = __builtin_fma((double)v[e + 1], (double)v[e + 1], s1);
      }
    }
    const int rest = count / U::N * U::N + threadIdx.x;
    if (rest < count) {
      const double v = (double)(float)p[rest];
      s0 = __builtin_fma(v, v, s0);
    }
  } else {
    for (int i = threadIdx.x; i < count; i += kGradThreads) {
      const double v = (double)(float)p[i];
      s0 = __builtin_fma(v, v, s0);
    }
  }
  return s0 + s1;
}

// the sum over the workgroup, in its first thread
__device__ __forceinline__ double group_sum(double x, double* s_part) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
  if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x == 0)
    for (unsigned w = 1; w < blockDim.x / 64; ++w) x += s_part[w];
  return x;
}

__global__ __launch_bounds__(kGradThreads) void grad_squares_kernel(const GradChunk* __restrict__ plan, int64_t chunks, double* __restrict__ partial) {
  __shared__ double s_part[kGradThreads / 64];
  double sum = 0.0;
  GradChunk next = plan[blockIdx.x];
  for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const GradChunk k = next;
    if (c + gridDim.x < chunks) next = plan[c + gridDim.x];
    if (k.bf16) sum += chunk_squares(static_cast<const __bf16*>(k.from), k.count);
    else sum += chunk_squares(static_cast<const float*>(k.from), k.count);
  }
  sum = group_sum(sum, s_part);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void grad_join_kernel(const double* __restrict__ partial, int n, double* __restrict__ sum) {
  __shared__ double s_part[16];
  double x = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 1024) x += partial[i];
  x = group_sum(x, s_part);
  if (threadIdx.x == 0) *sum = x;
}

constexpr int kPast = 2;      // the non-temporal bit of a buffer access
template <class T>
__device__ __forceinline__ void chunk_scale(const T* p, T* q, int count, float c) {
  using U = Unit<T>;
  constexpr int TURNS = KNAP_GRAD_CHUNK / (U::N * kGradThreads);
  if (((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & 15) == 0) {
    const uint32_t bytes = (uint32_t)count / U::N * 16u;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, bytes), w = make_rsrc(q, bytes);
    u32x4 x[TURNS];
#pragma unroll
    for (int i = 0; i < TURNS; ++i) x[i] = __builtin_amdgcn_raw_buffer_load_b128(r, (int)((threadIdx.x + i * kGradThreads) * 16u), 0, kPast);
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      float v[U::N];
      U::open(x[i], v);
#pragma unroll
      for (int e = 0; e < U::N; ++e) v[e] *= c;
      __builtin_amdgcn_raw_buffer_store_b128(U::close(v), w, (int)((threadIdx.x + i * kGradThreads) * 16u), 0, kPast);
    }
    const int rest = count / U::N * U::N + threadIdx.x;
    if (rest < count) q[rest] = (T)((float)p[rest] * c);
  } else {
    for (int i = threadIdx.x; i < count; i += kGradThreads) q[i] = (T)((float)p[i] * c);
  }
}

__global__ __launch_bounds__(kGradThreads) void grad_clip_kernel(const GradChunk* __restrict__ plan, int64_t chunks, const double* __restrict__ sum,
                                                                 float max_norm, float eps, float* norm) {
  const double length = sqrt(*sum);
  const double q = (double)max_norm / (length + (double)eps);
  // a NaN stays one; no limit clips nothing, whatever the norm
  const float c = q >= 1.0 || max_norm > 3.4028234e38f ? 1.f : (float)q;
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)length;
  if (blockIdx.x >= chunks) return;
  GradChunk next = plan[chunks - 1 - blockIdx.x];
  for (int64_t i = blockIdx.x; i < chunks; i += gridDim.x) {
    const GradChunk k = next;
    if (i + gridDim.x < chunks) next = plan[chunks - 1 - i - gridDim.x];
    if (c == 1.f && k.from == k.to) continue;
    if (k.bf16) chunk_scale(static_cast<const __bf16*>(k.from), static_cast<__bf16*>(k.to), k.count, c);
    else chunk_scale(static_cast<const float*>(k.from), static_cast<float*>(k.to), k.count, c);
  }
}

hipError_t launch_grad_squares(const GradChunk* plan, int64_t chunks, double* partial, double* sum, int cus, hipStream_t stream) {
  const int groups = (int)std::min<int64_t>(chunks, std::min(4 * cus, kGradGroups));
  if (groups > 0) {
    hipLaunchKernelGGL(grad_squares_kernel, dim3(groups), dim3(kGradThreads), 0, stream, plan, chunks, partial);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(grad_join_kernel, dim3(1), dim3(1024), 0, stream, partial, groups, sum);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradChunk* plan, int64_t chunks, const double* sum, float max_norm, float eps, float* norm, int cus, hipStream_t stream) {
  const int groups = (int)std::max<int64_t>(1, std::min<int64_t>(chunks, 8 * cus));
  hipLaunchKernelGGL(grad_clip_kernel, dim3(groups), dim3(kGradThreads), 0, stream, plan, chunks, sum, max_norm, eps, norm);
  return hipGetLastError();
}

}  // namespace knap
