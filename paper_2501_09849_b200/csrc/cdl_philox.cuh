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
// The same with the ten round keys made by the host: as kernel parameters they are operands of the rounds' logic instructions,
// where the sums cost two more instructions a round.
struct PhiloxKeys {
    unsigned int k0[10], k1[10];
};
inline PhiloxKeys philox_keys(unsigned long long seed)
{
    PhiloxKeys k;
    for (unsigned int r = 0; r < 10; ++r) {
        k.k0[r] = (unsigned int)seed + r * 0x9E3779B9u;
        k.k1[r] = (unsigned int)(seed >> 32) + r * 0xBB67AE85u;
    }
    return k;
}
// M0 times the first word of round 1, which (the counter's upper half being 0) is the block's high word ^ k0[0]: the same for
// 2^32 consecutive blocks, so a caller that draws many of them makes it once.
__device__ __forceinline__ unsigned long long philox_head(unsigned int block_hi, const PhiloxKeys &key)
{
    return (unsigned long long)0xD2511F53u * (block_hi ^ key.k0[0]);
}
__device__ __forceinline__ uint4 philox4x32_10(unsigned int block_lo, unsigned long long head, const PhiloxKeys &key)
{
    const unsigned int M0 = 0xD2511F53u, M1 = 0xCD9E8D57u;
    unsigned long long p = (unsigned long long)M0 * block_lo;                                       // round 0
    unsigned long long q = (unsigned long long)M1 * ((unsigned int)(p >> 32) ^ key.k1[0]);          // round 1
    unsigned int c0 = (unsigned int)(q >> 32) ^ key.k0[1], c1 = (unsigned int)q;
    unsigned int c2 = (unsigned int)(head >> 32) ^ (unsigned int)p ^ key.k1[1], c3 = (unsigned int)head;
#pragma unroll
    for (int r = 2; r < 10; ++r) {
        p = (unsigned long long)M0 * c0;
        q = (unsigned long long)M1 * c2;
        c0 = (unsigned int)(q >> 32) ^ c1 ^ key.k0[r];
        c1 = (unsigned int)q;
        c2 = (unsigned int)(p >> 32) ^ c3 ^ key.k1[r];
        c3 = (unsigned int)p;
    }
    return make_uint4(c0, c1, c2, c3);
}
__device__ __forceinline__ uint4 philox4x32_10(unsigned long long block, const PhiloxKeys &key)
{
    return philox4x32_10((unsigned int)block, philox_head((unsigned int)(block >> 32), key), key);
}
// top 24 bits of a word as a uniform number in [0, 1)
__device__ __forceinline__ float u01(unsigned int w) { return (float)(w >> 8) * 5.9604644775390625e-8f; }

}  // namespace cdl
