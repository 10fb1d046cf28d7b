// Stores past the caches, for the streaming operators.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace veda {

// 16 bytes that no later instruction of the kernel reads: not kept in the die's L2, where they would only push out what is still
// to be read.
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
__device__ __forceinline__ void store_through(void* p, uint4 v) {
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(p));
}

}  // namespace veda
