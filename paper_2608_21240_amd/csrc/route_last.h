// The last of a group of blocks of one launch to finish, without a fence (internal linkage: each source
// that includes it compiles its own copy).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spice {
namespace {

// The last of a token's routing blocks to finish, found with an arrival counter.  A block's
// logits are agent-scope stores (written through to the device-coherent level), so ordering
// them before its increment needs only that every wave's stores have completed (s_waitcnt
// vmcnt(0)), not an L2 write-back; the last block reads them with agent-scope loads, not
// after an L2 invalidate.  Neither disturbs the tiles that stream beside the routing
// blocks.  The last block resets the counter, so it is zero again for the next call.
__device__ __forceinline__ bool route_last_block(uint32_t* counter, uint32_t n_blocks, int* s_flag) {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's stores have completed
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t prev = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const bool last = prev == n_blocks - 1;
        if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *s_flag = last ? 1 : 0;
    }
    __syncthreads();
    return *s_flag != 0;
}

}  // namespace
}  // namespace spice
