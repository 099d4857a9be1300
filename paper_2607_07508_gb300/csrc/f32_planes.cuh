// Three bf16 pieces of an fp32 value, and the classes of magnitude that decide whether
// a product may use them (see logprobs_f32.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

namespace sao {

constexpr float CLASS_LIMIT[3] = {0x1p26f, 0x1p62f, 0x1p100f};
// a = p0 + p1 + p2, for |a| below 2^100
__device__ __forceinline__ void split3(float a, float &p0, float &p1, float &p2) {
  p0 = __bfloat162float(__float2bfloat16_rn(a));
  const float r = a - p0;
  p1 = __bfloat162float(__float2bfloat16_rn(r));
  p2 = r - p1;
}
// Largest magnitude (NaN if there is one), and its class.
__device__ __forceinline__ float larger(float most, float a) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(most), "f"(fabsf(a)));
  return r;
}
__device__ __forceinline__ void raise_class(unsigned int *word, float most) {
  const unsigned c = !(most < CLASS_LIMIT[0]) + !(most < CLASS_LIMIT[1]) + !(most < CLASS_LIMIT[2]);
  if (c > 0) atomicMax(word, c);
}

}  // namespace sao
