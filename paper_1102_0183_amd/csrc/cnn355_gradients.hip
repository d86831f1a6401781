// The 2-norm of all gradients of a step, gradients clipped by it, and the update with clipped gradients:
//
//   N = sqrt(sum over tensors, elements of g^2),  f = max_norm / N where N > max_norm, else 1
//   clipped: g f        update: w - lr f g        (N infinite or no number: g, and w, as they are)
//
// Two launches: every workgroup of the first leaves the sum of its chunks in memory, every workgroup of the second adds all
// those sums (the same way, so that all agree on N to the last bit and a call gives the same bits again) and goes over its
// chunks.  Squares and sums are doubles: no gradient that a float holds overflows or vanishes in its square, and the order of
// a thousand million terms does not show.  So is the product with the factor, which is rounded once.
#include <hip/hip_runtime.h>

#include <algorithm>

#define CNN_GLOBAL __attribute__((address_space(1)))
#include "cnn355_ops.h"
#include "cnn355_elements.h"

namespace cnn355 {

namespace {

constexpr int GT = 256;   // threads of a workgroup

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));

// the sum of a double of every thread, in every thread
__device__ __forceinline__ double sum_of_workgroup(double s, double* lds) {
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) lds[wave] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < GT / 64; ++w) s += lds[w];
  return s;
}

// the tensor that chunk c is of
__device__ __forceinline__ int tensor_of(const TensorJob& J, unsigned c) {
  int lo = 0, hi = J.tensors;   // chunk[lo] <= c < chunk[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (J.chunk[mid] <= c) lo = mid; else hi = mid;
  }
  return lo;
}

// ---- the sum of squares ----
template <int TYPE>
__device__ __forceinline__ double squares(const CNN_GLOBAL void* from, unsigned long long begin, unsigned long long n) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  constexpr int V = E::V, N = LIST_CHUNK / GT / V;
  const CNN_GLOBAL T* g = (const CNN_GLOBAL T*)from + begin;
  double s = 0.0;
  if (n - begin >= LIST_CHUNK) {
    v4u r[N];
#pragma unroll
    for (int q = 0; q < N; ++q) r[q] = *(const CNN_GLOBAL v4u_any*)(g + (q * GT + threadIdx.x) * V);
#pragma unroll
    for (int q = 0; q < N; ++q)
#pragma unroll
      for (int j = 0; j < V; ++j) { const double v = E::get(r[q], j); s = fma(v, v, s); }
    return s;
  }
  const int left = (int)(n - begin), whole = left / V;
  for (int i = threadIdx.x; i < whole; i += GT) {
    const v4u r = *(const CNN_GLOBAL v4u_any*)(g + i * V);
#pragma unroll
    for (int j = 0; j < V; ++j) { const double v = E::get(r, j); s = fma(v, v, s); }
  }
  const int last = whole * V + (int)threadIdx.x;
  if (last < left) { const double v = E::get(g[last]); s = fma(v, v, s); }
  return s;
}

__global__ void __launch_bounds__(GT) k_squares(TensorJob J, CNN_GLOBAL double* sums) {
  __shared__ double lds[GT / 64];
  double s = 0.0;
  for (unsigned c = blockIdx.x; c < J.chunks; c += gridDim.x) {
    const int t = tensor_of(J, c);
    const unsigned long long begin = (unsigned long long)(c - J.chunk[t]) * LIST_CHUNK;
    switch (J.type[t]) {
      case ELEMENT_F32: s += squares<ELEMENT_F32>(J.from[t], begin, J.n[t]); break;
      case ELEMENT_BF16: s += squares<ELEMENT_BF16>(J.from[t], begin, J.n[t]); break;
      default: s += squares<ELEMENT_F16>(J.from[t], begin, J.n[t]); break;
    }
  }
  s = sum_of_workgroup(s, lds);
  if (threadIdx.x == 0) sums[J.first_sum + blockIdx.x] = s;
}

__device__ __forceinline__ double norm_of(const CNN_GLOBAL double* sums, int n, double* lds) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += GT) s += sums[i];
  return sqrt(sum_of_workgroup(s, lds));
}

__global__ void __launch_bounds__(GT) k_norm(const CNN_GLOBAL double* sums, int n, CNN_GLOBAL float* norm) {
  __shared__ double lds[GT / 64];
  const double v = norm_of(sums, n, lds);
  if (threadIdx.x == 0) *norm = (float)v;
}

// ---- what is done with it ----
template <int TYPE>
__device__ __forceinline__ void scale(const CNN_GLOBAL void* from, CNN_GLOBAL void* to, unsigned long long begin, unsigned long long n, double f) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  constexpr int V = E::V, N = LIST_CHUNK / GT / V;
  const CNN_GLOBAL T* g = (const CNN_GLOBAL T*)from + begin;
  CNN_GLOBAL T* o = (CNN_GLOBAL T*)to + begin;
  auto one = [&](float v) { return E::make((float)(v * f)); };
  auto sixteen = [&](v4u r) {
    union { v4u v; T e[V]; } out;
#pragma unroll
    for (int j = 0; j < V; ++j) out.e[j] = one(E::get(r, j));
    return out.v;
  };
  if (n - begin >= LIST_CHUNK) {
    v4u r[N];
#pragma unroll
    for (int q = 0; q < N; ++q) r[q] = *(const CNN_GLOBAL v4u_any*)(g + (q * GT + threadIdx.x) * V);
#pragma unroll
    for (int q = 0; q < N; ++q) *(CNN_GLOBAL v4u_any*)(o + (q * GT + threadIdx.x) * V) = sixteen(r[q]);
    return;
  }
  const int left = (int)(n - begin), whole = left / V;
  for (int i = threadIdx.x; i < whole; i += GT) *(CNN_GLOBAL v4u_any*)(o + i * V) = sixteen(*(const CNN_GLOBAL v4u_any*)(g + i * V));
  const int last = whole * V + (int)threadIdx.x;
  if (last < left) o[last] = one(E::get(g[last]));
}

template <int TYPE>
__device__ __forceinline__ void update(const CNN_GLOBAL void* from, CNN_GLOBAL void* to, unsigned long long begin, unsigned long long n, double f) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  constexpr int V = E::V, N = LIST_CHUNK / GT / V, W = V / 4;
  const CNN_GLOBAL T* g = (const CNN_GLOBAL T*)from + begin;
  CNN_GLOBAL float* w = (CNN_GLOBAL float*)to + begin;
  auto one = [&](float w, float g) { return (float)fma(-f, (double)g, (double)w); };
  auto some = [&](int at, v4u r, const v4f (&v)[W]) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      v4f o;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = one(v[k][j], E::get(r, 4 * k + j));
      *(CNN_GLOBAL v4f_any*)(w + at + 4 * k) = o;
    }
  };
  const int left = n - begin < LIST_CHUNK ? (int)(n - begin) : LIST_CHUNK, whole = left / V;
  if (left == LIST_CHUNK) {
    constexpr int B = N < 4 ? N : 4;   // (loads that wait together)
#pragma unroll 1
    for (int q0 = 0; q0 < N; q0 += B) {
      v4u r[B];
      v4f v[B][W];
#pragma unroll
      for (int q = 0; q < B; ++q) {
        const int at = ((q0 + q) * GT + threadIdx.x) * V;
        r[q] = *(const CNN_GLOBAL v4u_any*)(g + at);
#pragma unroll
        for (int k = 0; k < W; ++k) v[q][k] = *(const CNN_GLOBAL v4f_any*)(w + at + 4 * k);
      }
#pragma unroll
      for (int q = 0; q < B; ++q) some(((q0 + q) * GT + threadIdx.x) * V, r[q], v[q]);
    }
    return;
  }
  for (int i = threadIdx.x; i < whole; i += GT) {
    const v4u r = *(const CNN_GLOBAL v4u_any*)(g + i * V);
    v4f v[W];
#pragma unroll
    for (int k = 0; k < W; ++k) v[k] = *(const CNN_GLOBAL v4f_any*)(w + i * V + 4 * k);
    some(i * V, r, v);
  }
  const int last = whole * V + (int)threadIdx.x;
  if (last < left) w[last] = one(w[last], E::get(g[last]));
}

// UPDATE: to holds weights (float), `lr` is the rate; else to holds the clipped gradients, which may be `from` themselves.
template <bool UPDATE>
__global__ void __launch_bounds__(GT) k_apply(TensorJob J, const CNN_GLOBAL double* sums, double max_norm, double lr, CNN_GLOBAL float* norm, int in_place) {
  __shared__ double lds[GT / 64];
  const double v = norm_of(sums, J.sums, lds);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
  const bool finite = v < __builtin_inf();
  double f = finite && v > max_norm ? max_norm / v : 1.0;
  if (UPDATE) {
    if (!finite) return;
    f *= lr;
  } else if (in_place && f == 1.0) {
    return;
  }
  // the last chunks first: they are the ones that the first launch read last, and may still be in the cache
  for (unsigned k = blockIdx.x; k < J.chunks; k += gridDim.x) {
    const unsigned c = J.chunks - 1 - k;
    const int t = tensor_of(J, c);
    const unsigned long long begin = (unsigned long long)(c - J.chunk[t]) * LIST_CHUNK;
    if (UPDATE) {
      switch (J.type[t]) {
        case ELEMENT_F32: update<ELEMENT_F32>(J.from[t], J.to[t], begin, J.n[t], f); break;
        case ELEMENT_BF16: update<ELEMENT_BF16>(J.from[t], J.to[t], begin, J.n[t], f); break;
        default: update<ELEMENT_F16>(J.from[t], J.to[t], begin, J.n[t], f); break;
      }
    } else {
      switch (J.type[t]) {
        case ELEMENT_F32: scale<ELEMENT_F32>(J.from[t], J.to[t], begin, J.n[t], f); break;
        case ELEMENT_BF16: scale<ELEMENT_BF16>(J.from[t], J.to[t], begin, J.n[t], f); break;
        default: scale<ELEMENT_F16>(J.from[t], J.to[t], begin, J.n[t], f); break;
      }
    }
  }
}

constexpr unsigned APPLY_GRID = 2048;

}  // namespace

hipError_t launch_squares(hipStream_t stream, const TensorJob& J, int workgroups, double* sums) {
  hipLaunchKernelGGL(k_squares, dim3((unsigned)workgroups), dim3(GT), 0, stream, J, (CNN_GLOBAL double*)sums);
  return hipGetLastError();
}

hipError_t launch_norm(hipStream_t stream, const double* sums, int n, float* norm) {
  hipLaunchKernelGGL(k_norm, dim3(1), dim3(GT), 0, stream, (const CNN_GLOBAL double*)sums, n, (CNN_GLOBAL float*)norm);
  return hipGetLastError();
}

hipError_t launch_scale(hipStream_t stream, const TensorJob& J, const double* sums, double max_norm, float* norm, int in_place) {
  hipLaunchKernelGGL(k_apply<false>, dim3(std::max(1u, std::min(J.chunks, APPLY_GRID))), dim3(GT), 0, stream, J, (const CNN_GLOBAL double*)sums, max_norm, 0.0,
                     (CNN_GLOBAL float*)norm, in_place);
  return hipGetLastError();
}

hipError_t launch_update(hipStream_t stream, const TensorJob& J, const double* sums, double max_norm, double lr, float* norm) {
  hipLaunchKernelGGL(k_apply<true>, dim3(std::max(1u, std::min(J.chunks, APPLY_GRID))), dim3(GT), 0, stream, J, (const CNN_GLOBAL double*)sums, max_norm, lr,
                     (CNN_GLOBAL float*)norm, 0);
  return hipGetLastError();
}

}  // namespace cnn355
