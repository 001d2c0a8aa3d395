// The counter-based generator of the sampling quantizer and of dropout.
#pragma once
#include <stdint.h>

namespace cdl {

// Philox4x32-10 (Salmon et al., SC 2011) from its definition: ten rounds of
//   (c0,c1,c2,c3) <- (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)),  key += (W0, W1) between rounds.
// Counter = (block number, 0), key = seed; the block's four words serve elements 4 b .. 4 b + 3.
__device__ __forceinline__ uint4 philox4x32_10(unsigned long long block, unsigned long long seed)
{
    const unsigned int M0 = 0xD2511F53u, M1 = 0xCD9E8D57u, W0 = 0x9E3779B9u, W1 = 0xBB67AE85u;
    unsigned int c0 = (unsigned int)block, c1 = (unsigned int)(block >> 32), c2 = 0u, c3 = 0u;
    unsigned int k0 = (unsigned int)seed, k1 = (unsigned int)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        if (r > 0) {
            k0 += W0;
            k1 += W1;
        }
        const unsigned int n0 = __umulhi(M1, c2) ^ c1 ^ k0;
        const unsigned int n1 = M1 * c2;
        const unsigned int n2 = __umulhi(M0, c0) ^ c3 ^ k1;
        const unsigned int n3 = M0 * c0;
        c0 = n0;
        c1 = n1;
        c2 = n2;
        c3 = n3;
    }
    return make_uint4(c0, c1, c2, c3);
}
// top 24 bits of a word as a uniform number in [0, 1)
__device__ __forceinline__ float u01(unsigned int w) { return (float)(w >> 8) * 5.9604644775390625e-8f; }

}  // namespace cdl
