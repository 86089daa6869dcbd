// Philox4x32-10 (Salmon et al., SC'11): four 32-bit numbers from a counter of four words and a key of two.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hadfl {

struct U4 { uint32_t x, y, z, w; };

__device__ __forceinline__ U4 philox4x32_10(U4 c, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
        c = U4{(uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a};
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    return c;
}

}  // namespace hadfl
