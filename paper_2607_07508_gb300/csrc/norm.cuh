// Root-mean-square norm (norm.cu), for the C entry points.
#pragma once

#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include "../../include/sao.h"

namespace sao {

struct NormFwd {
  const void *x, *residual;  // residual, sum: or null
  const void *weight;
  void *sum, *y;             // y: or null
  float *rstd;               // or null
  uint8_t *y8;               // or null
  void *scales;
  int scaling;
  float eps;
  int64_t N;
  int h;
};
struct NormBwd {
  const void *x, *weight;
  const float *rstd;
  const void *dy, *dsum;     // dsum: or null
  void *dx;
  float *dweight;            // or null
  int accumulate;
  int64_t N;
  int h;
};

namespace norm {

// The maximum, NaN if one of them is (an 8-bit scale that hides a NaN would be a number).
__device__ __forceinline__ float max_nan(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}

// Squares of values below 2^-63 lose digits in fp32, and vanish. Where eps does not hide that, a row whose mean of
// squares (with eps) is below kSmall is summed again, times kUp: its values are then 2^-49 to 2^57.
constexpr float kSmall = 0x1p-100f, kUp = 0x1p100f;

// A block's scale and what its values are multiplied by. amax / 448 is the largest e4m3 value's.
__device__ __forceinline__ float scale_of(float amax, float *inverse) {
  const float s = max_nan(amax / 448.f, FLT_MIN);  // a block of zeros has a scale all the same
  *inverse = 1.f / s;
  return s;
}
// The least power of two 2^(b - 127) that amax / 448 does not pass (b = 255: NaN). 448 is 1.75 2^8: the exponent less 8,
// and one more where the mantissa is past 1.75.
__device__ __forceinline__ uint32_t power_of(float amax, float *inverse) {
  const uint32_t u = __float_as_uint(amax);
  const int e = int((u + 0x1fffffu) >> 23) - 8;
  const uint32_t b = u >= 0x7f800000u ? 255u : e > 0 ? uint32_t(e) : 0u;
  *inverse = b == 255u ? NAN : __uint_as_float((254u - b) << 23);
  return b;
}

}  // namespace norm

size_t norm_ws_bytes(int64_t N, int32_t h);
sao_status norm_fwd_launch(const NormFwd &a, sao_dtype dt, sao_dtype w_dt, cudaStream_t s);
sao_status norm_bwd_launch(const NormBwd &a, sao_dtype dt, sao_dtype w_dt, void *ws, size_t ws_bytes, cudaStream_t s);

// norm_tiles.cu: the same, arrays on 16 bytes; the forward for rows of any length, the backward for those of up to
// kShortRow. The backward has at most `most` CTAs, and writes how many (`parts`) have sums for dw in `partial`.
constexpr int kShortRow = 64;
sao_status norm_fwd_tiles_launch(const NormFwd &a, sao_dtype dt, sao_dtype w_dt, cudaStream_t s);
sao_status norm_bwd_tiles_launch(const NormBwd &a, sao_dtype dt, sao_dtype w_dt, float *partial, int most, int *parts,
                                 cudaStream_t s);

}  // namespace sao
