// Global norm of many gradients and clipping by it:
//   S = sum g^2 over all tensors,  c = min(1, max_norm / (sqrt(S) + eps)),  out = c g.
// Bound by HBM: every gradient is read once for S and once more for the product, which is written once.  A launch takes a table of tensors
// in its arguments, so that nothing is copied to the device before it; its workgroups take chunks of kGradChunk elements in turn and look
// up whose they are.  Squares and sums are in 64 bits (of which the card does as many as of 32): no gradient that is finite overflows or
// vanishes in them, and the norm is right to its last bit in 32.  Every workgroup leaves one sum, which a second launch adds up in a fixed order.
#include "knap_device.h"
#include "knap_kernels.h"

namespace knap {

constexpr int kGradThreads = 256;

// the tensor that chunk c belongs to
__device__ __forceinline__ int tensor_of(const GradTable& t, uint32_t c) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= c) lo = mid; else hi = mid - 1;
  }
  return lo;
}

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
  constexpr int TURNS = kGradChunk / (U::N * kGradThreads);
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

__global__ __launch_bounds__(kGradThreads) void grad_squares_kernel(GradTable t, double* partial) {
  __shared__ double s_part[kGradThreads / 64];
  double sum = 0.0;
  const uint32_t chunks = t.first[t.n];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int i = tensor_of(t, c);
    const int64_t start = (int64_t)(c - t.first[i]) * kGradChunk;
    const int count = (int)min((int64_t)kGradChunk, t.numel[i] - start);
    if (t.bf16[i]) sum += chunk_squares(static_cast<const __bf16*>(t.from[i]) + start, count);
    else sum += chunk_squares(static_cast<const float*>(t.from[i]) + start, count);
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

template <class T>
__device__ __forceinline__ void chunk_scale(const T* p, T* q, int count, float c) {
  using U = Unit<T>;
  constexpr int TURNS = kGradChunk / (U::N * kGradThreads);
  if (((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & 15) == 0) {
    const uint32_t bytes = (uint32_t)count / U::N * 16u;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, bytes), w = make_rsrc(q, bytes);
    u32x4 x[TURNS];
#pragma unroll
    for (int i = 0; i < TURNS; ++i) x[i] = buffer_load16(r, (threadIdx.x + i * kGradThreads) * 16u);
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
      float v[U::N];
      U::open(x[i], v);
#pragma unroll
      for (int e = 0; e < U::N; ++e) v[e] *= c;
      __builtin_amdgcn_raw_buffer_store_b128(U::close(v), w, (int)((threadIdx.x + i * kGradThreads) * 16u), 0, 0);
    }
    const int rest = count / U::N * U::N + threadIdx.x;
    if (rest < count) q[rest] = (T)((float)p[rest] * c);
  } else {
    for (int i = threadIdx.x; i < count; i += kGradThreads) q[i] = (T)((float)p[i] * c);
  }
}

__global__ __launch_bounds__(kGradThreads) void grad_clip_kernel(GradTable t, const double* __restrict__ sum, float max_norm, float eps, float* norm) {
  const double length = sqrt(*sum);
  const double q = (double)max_norm / (length + (double)eps);
  // a NaN stays one; no limit clips nothing, whatever the norm
  const float c = q >= 1.0 || max_norm > 3.4028234e38f ? 1.f : (float)q;
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)length;
  const uint32_t chunks = t.first[t.n];
  for (uint32_t k = blockIdx.x; k < chunks; k += gridDim.x) {
    const int i = tensor_of(t, k);
    if (c == 1.f && t.from[i] == t.to[i]) continue;
    const int64_t start = (int64_t)(k - t.first[i]) * kGradChunk;
    const int count = (int)min((int64_t)kGradChunk, t.numel[i] - start);
    if (t.bf16[i]) chunk_scale(static_cast<const __bf16*>(t.from[i]) + start, static_cast<__bf16*>(t.to[i]) + start, count, c);
    else chunk_scale(static_cast<const float*>(t.from[i]) + start, static_cast<float*>(t.to[i]) + start, count, c);
  }
}

hipError_t launch_grad_squares(const GradTable& t, double* partial, int groups, hipStream_t stream) {
  hipLaunchKernelGGL(grad_squares_kernel, dim3(groups), dim3(kGradThreads), 0, stream, t, partial);
  return hipGetLastError();
}
hipError_t launch_grad_join(const double* partial, int n, double* sum, hipStream_t stream) {
  hipLaunchKernelGGL(grad_join_kernel, dim3(1), dim3(1024), 0, stream, partial, n, sum);
  return hipGetLastError();
}
hipError_t launch_grad_clip(const GradTable& t, const double* sum, float max_norm, float eps, float* norm, int groups, hipStream_t stream) {
  hipLaunchKernelGGL(grad_clip_kernel, dim3(groups), dim3(kGradThreads), 0, stream, t, sum, max_norm, eps, norm);
  return hipGetLastError();
}

}  // namespace knap
