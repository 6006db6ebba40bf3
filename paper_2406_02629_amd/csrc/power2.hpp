// Weights of a softmax in whole numbers, shared by the attention kernels and by those that draw tokens.
#pragma once
#include "field.hpp"

namespace SS_NS {

// floor(2^30 2^-x) for x in octaves with 16 fraction bits: 2^-x for x in [0, 1) by a polynomial of degree 5 that takes the value 1 at 0 and
// is off by 2.2e-7 at most, Horner's scheme in 30 fraction bits, each product cut to them
__device__ __forceinline__ u32 power2(u64 x)
{
    const u32 r = (u32)x << 16;                  // the fraction, 32 bits
    u32 w = 1077640u;
    w = 10033292u - __umulhi(w, r);
    w = 59494488u - __umulhi(w, r);
    w = 257928559u - __umulhi(w, r);
    w = 744260865u - __umulhi(w, r);
    w = 1073741824u - __umulhi(w, r);
    const u64 octaves = x >> 16;
    return octaves < 31 ? w >> octaves : 0;
}

}  // namespace SS_NS
