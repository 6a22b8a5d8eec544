// The counter-based generator of every random draw in this library.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sparcml {

// Philox4x32-10 (Salmon et al., SC'11): ten rounds of two 32x32->64
// multiplies with the high halves mixed into the other words and the key,
// the key advanced by the Weyl constants between rounds.
__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        if (i) {
            k0 += 0x9E3779B9u;
            k1 += 0xBB67AE85u;
        }
        // full 64-bit products: one v_mad_u64_u32 each instead of a low and
        // a high multiply
        const uint64_t p0 = (uint64_t)0xD2511F53u * c.x, p1 = (uint64_t)0xCD9E8D57u * c.z;
        const uint32_t lo0 = (uint32_t)p0, hi0 = (uint32_t)(p0 >> 32);
        const uint32_t lo1 = (uint32_t)p1, hi1 = (uint32_t)(p1 >> 32);
        c = make_uint4(hi1 ^ c.y ^ k0, lo1, hi0 ^ c.w ^ k1, lo0);
    }
    return c;
}

}  // namespace sparcml
