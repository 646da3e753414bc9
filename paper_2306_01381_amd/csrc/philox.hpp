// Philox4x32-10 (Salmon et al., SC'11).  The key schedule is wave-uniform (it only depends on the seed).
#pragma once

#include "common.hpp"

namespace adaqp {

struct Rand128 { uint32_t w0, w1, w2, w3; };

// a ^ b ^ c in one instruction: gfx950's v_bitop3_b32 with the truth table of the three-input xor (the compiler
// does not form it from two xors)
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c)
{
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}

__device__ __forceinline__ Rand128 philox4x32_10(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3,
                                                 uint32_t k0, uint32_t k1)
{
    constexpr uint32_t kMulA = 0xD2511F53u, kMulB = 0xCD9E8D57u;
    constexpr uint32_t kWeylA = 0x9E3779B9u, kWeylB = 0xBB67AE85u;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t pA = (uint64_t)kMulA * c0;            // one v_mad_u64_u32 each
        const uint64_t pB = (uint64_t)kMulB * c2;
        c0 = xor3((uint32_t)(pB >> 32), c1, k0);
        c1 = (uint32_t)pB;
        c2 = xor3((uint32_t)(pA >> 32), c3, k1);
        c3 = (uint32_t)pA;
        k0 += kWeylA;
        k1 += kWeylB;
    }
    return Rand128{c0, c1, c2, c3};
}

}  // namespace adaqp
