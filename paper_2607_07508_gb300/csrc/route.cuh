// Routing to experts (route.cu), for the C entry points.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sao.h"

namespace sao {

struct RouteArgs {
  const void *x;          // [N, E]
  const float *bias;      // or null
  const uint8_t *mask;    // or null
  int64_t N;
  int E, k, score;
  int groups, kept, two;  // groups of experts, those that stay, by the sum of their best two
  int renorm;
  float scale;
  int replay;
  int32_t *ids;
  float *weights;
  unsigned int *err;
};
struct RouteBwdArgs {
  const void *x;
  const uint8_t *mask;
  int64_t N;
  int E, k, score, renorm;
  float scale;
  const int32_t *ids;
  const float *weights, *grad;
  void *dx;
  int accumulate;
  unsigned int *err;
};

sao_status route_fwd_launch(const RouteArgs &a, sao_dtype dt, cudaStream_t s);
sao_status route_bwd_launch(const RouteBwdArgs &a, sao_dtype dt, cudaStream_t s);

}  // namespace sao
