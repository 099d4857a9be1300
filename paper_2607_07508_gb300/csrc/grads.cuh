// Global norm and clipping of gradients (grads.cu), for the C entry points.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sao.h"

namespace sao {

size_t grad_ws_bytes();
// Refuses tensors that share a byte, but for an out[i] that is grads[i] (out may be null).
sao_status check_disjoint(const sao_tensor *grads, const sao_tensor *out, int32_t count);
sao_status grad_sumsq_launch(const sao_tensor *grads, int32_t count, double *sumsq, void *ws, size_t ws_bytes,
                             cudaStream_t s);
sao_status grad_clip_launch(const sao_tensor *grads, const sao_tensor *out, int32_t count, const double *sumsq,
                            float max_norm, float *norm, float *coef, cudaStream_t s);

}  // namespace sao
