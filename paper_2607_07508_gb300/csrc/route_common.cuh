// Shared by the routing kernels.
#pragma once

#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "route.cuh"
#include "sao_common.cuh"
#include "sao_internal.h"

namespace sao {
namespace route {

constexpr int kWarps = 8;  // of a CTA of the forward
constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ float value(const float *p) { return ld(p); }
__device__ __forceinline__ float value(const __nv_bfloat16 *p) {
  return __uint_as_float(uint32_t(ld(reinterpret_cast<const uint16_t *>(p))) << 16);
}

template <class F>
__device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

__device__ __forceinline__ float exp_of(float v) { return expf(v); }
__device__ __forceinline__ double exp_of(double v) { return exp(v); }
template <class F>
__device__ __forceinline__ F sigmoid(F x) {
  const F e = exp_of(-fabs(x));  // never past the range, and small scores keep their digits
  return (x < F(0) ? e : F(1)) / (F(1) + e);
}

// The sum of exp(x - top) over n logits from p on, in kParts (a power of two) chains of additions. (One chain of 128 was
// off by 126 units of 2^-24 where each addition is rounded the same way.)
template <int kParts, class T>
__device__ __forceinline__ float sum_of_exponentials(const T *p, int n, float top) {
  float part[kParts] = {};
  int e = 0;
#pragma unroll 1
  for (; e + kParts <= n; e += kParts)
#pragma unroll
    for (int i = 0; i < kParts; ++i) part[i] += expf(value(p + e + i) - top);
#pragma unroll
  for (int i = 0; i < kParts - 1; ++i)
    if (e + i < n) part[i] += expf(value(p + e + i) - top);
#pragma unroll
  for (int o = kParts / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < o; ++i) part[i] += part[i + o];
  return part[0];
}

// Over the k lanes from `first` on, a multiple of k (`even`: k is a power of two).
__device__ __forceinline__ float share_sum(float v, int first, int k, bool even) {
  if (even) {
    for (int o = k >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
  }
  float s = 0.f;
#pragma unroll 2
  for (int i = 0; i < k; ++i) s += __shfl_sync(kAll, v, first + i);
  return s;
}
__device__ __forceinline__ float share_max(float v, int first, int k, bool even) {
  if (even) {
    for (int o = k >> 1; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
  }
  float m = -INFINITY;
#pragma unroll 2
  for (int i = 0; i < k; ++i) m = fmaxf(m, __shfl_sync(kAll, v, first + i));
  return m;
}

template <class F>
sao_status by_type(sao_dtype dt, F f) {
  return dt == SAO_BF16 ? f(__nv_bfloat16()) : f(float());
}

inline int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

}  // namespace route
}  // namespace sao
