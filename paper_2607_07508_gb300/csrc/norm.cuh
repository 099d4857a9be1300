// Root-mean-square norm (norm.cu), for the C entry points.
#pragma once

#include <cuda_runtime.h>
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

size_t norm_ws_bytes(int64_t N, int32_t h);
sao_status norm_fwd_launch(const NormFwd &a, sao_dtype dt, sao_dtype w_dt, cudaStream_t s);
sao_status norm_bwd_launch(const NormBwd &a, sao_dtype dt, sao_dtype w_dt, void *ws, size_t ws_bytes, cudaStream_t s);

// norm_tiles.cu: the same for rows of any length, arrays on 16 bytes, no 8-bit rows. The backward has at most
// `most` CTAs, and writes how many (`parts`) have sums for dw in `partial`.
sao_status norm_fwd_tiles_launch(const NormFwd &a, sao_dtype dt, sao_dtype w_dt, cudaStream_t s);
sao_status norm_bwd_tiles_launch(const NormBwd &a, sao_dtype dt, sao_dtype w_dt, float *partial, int most, int *parts,
                                 cudaStream_t s);

}  // namespace sao
