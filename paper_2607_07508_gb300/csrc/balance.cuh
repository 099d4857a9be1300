// Load-balance loss of a mixture of experts (balance.cu), for the C entry points.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sao.h"

namespace sao {

size_t balance_ws_bytes(int64_t N, int32_t E, int32_t B);
sao_status balance_fwd_launch(const void *x, sao_dtype dt, const int32_t *ids, const uint8_t *mask, const int32_t *cu,
                              int32_t B, int64_t N, int32_t E, int32_t k, int score, float *loss, int64_t *counts,
                              float *prob_sums, int64_t *rows, unsigned int *err, void *ws, size_t ws_bytes,
                              cudaStream_t s);
sao_status balance_bwd_launch(const void *x, sao_dtype dt, const uint8_t *mask, const int32_t *cu, int32_t B, int64_t N,
                              int32_t E, int32_t k, int score, const int64_t *counts, const int64_t *rows,
                              const float *grad_loss, void *dx, unsigned int *err, cudaStream_t s);

}  // namespace sao
