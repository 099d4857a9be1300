// Untiled bulk copies (cp.async.bulk) out of shared memory, and what goes with them.
#pragma once

#include <stdint.h>

#include "tc_ptx.cuh"

namespace sao {
namespace bulk {

// bytes: a multiple of 16; both addresses on 16 bytes. One thread issues it, after tc::fence_proxy_async_smem() by
// the threads that wrote and a barrier; tc::bulk_commit_group() and tc::bulk_wait_group*() by the same thread.
__device__ __forceinline__ void store(void *dst, const void *smem, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(tc::smem_u32(smem)),
               "r"(bytes)
               : "memory");
}

}  // namespace bulk
}  // namespace sao
