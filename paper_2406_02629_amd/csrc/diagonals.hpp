// Anti-diagonal sums of a product of balanced 8-bit digits, and the field element they stand for: shared by the kernels that multiply
// on int8 MFMA.
#pragma once
#include "field.hpp"

namespace SS_NS {

typedef int v4i __attribute__((ext_vector_type(4)));

// NL digits per field element (8 for p = 2^61 - 1, 6 for p = 2^45 - 55: the digits above are zero), hence
// ND anti-diagonal sums; a packed tile (16 rows x 64 contraction indices) is NL limb slices of 64 lanes x
// 16 bytes = TILE 16-byte words
constexpr int NL = SS_NLIMB, ND = 2 * NL - 1, TILE = NL * 64;

// a * b + c, one instruction (the compiler turns a multiplication by a power of two into a sign extension,
// a 64-bit shift and a 64-bit addition)
__device__ __forceinline__ long long mad_i64(int a, int b, long long c)
{
    long long d;
    asm("v_mad_i64_i32 %0, vcc, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c) : "vcc");
    return d;
}

// D_0 + D_1 2^8 + D_2 2^16 (+ D_3 2^24): up to four of the signed 32-bit diagonal sums in one signed 64-bit
// word, |result| < 2^31 (1 + 2^8 + 2^16 + 2^24) < 2^56
__device__ __forceinline__ long long join4(int d0, int d1, int d2, int d3)
{
    return mad_i64(d3, 1 << 24, mad_i64(d2, 1 << 16, mad_i64(d1, 1 << 8, (long long)d0)));
}
__device__ __forceinline__ long long join3(int d0, int d1, int d2)
{
    return mad_i64(d2, 1 << 16, mad_i64(d1, 1 << 8, (long long)d0));
}

// The ND diagonal sums of one output -> canonical field element.  The sums are signed 32-bit numbers and
// stay signed: four of them at a time go into one signed 64-bit word, the words are joined with the field's
// reduction rule, and a multiple of p makes the total positive before it is reduced.  `more` < 2^62 (2^47) is added on the way.
#if defined(SS_FIELD_P45)
__device__ __forceinline__ u64 fold_diagonals(const v4i (&acc)[ND], int r, u64 more = 0)
{
    const long long off = (long long)(SS_P << 12);   // a multiple of p above 2^56
    const u64 g0 = (u64)(join4(acc[0][r], acc[1][r], acc[2][r], acc[3][r]) + off);
    const u64 g1 = (u64)(join4(acc[4][r], acc[5][r], acc[6][r], acc[7][r]) + off);
    const u64 g2 = (u64)(join3(acc[8][r], acc[9][r], acc[10][r]) + off);
    // g0 + g1 2^32 + g2 2^64.  With g = a 2^13 + b: g 2^32 = a 2^45 + b 2^32 = 55 a + b 2^32, and
    // 2^64 = 55 2^19 (mod p)
    const u64 r1 = ss_reduce(g1), r2 = ss_reduce(g2);
    const u64 t1 = SS_PC * (r1 >> 13) + ((r1 & 0x1FFFull) << 32);   // < 2^38 + 2^45
    const u64 t2 = ss_mul(r2, SS_PC << 19);
    return ss_reduce(ss_fold(g0) + t1 + t2 + more);
}
#else
__device__ __forceinline__ u64 fold_diagonals(const v4i (&acc)[15], int r, u64 more = 0)
{
    const long long g0 = join4(acc[0][r], acc[1][r], acc[2][r], acc[3][r]);
    const long long g1 = join4(acc[4][r], acc[5][r], acc[6][r], acc[7][r]);
    const long long g2 = join4(acc[8][r], acc[9][r], acc[10][r], acc[11][r]);
    const long long g3 = join3(acc[12][r], acc[13][r], acc[14][r]);
    // g0 + g1 2^32 + g2 2^64 + g3 2^96 with 2^61 = 1: 2^64 = 2^3, 2^96 = 2^35 = 2^3 2^32
    const long long lo = g0 + (g2 << 3), hi = g1 + (g3 << 3);   // |.| < 2^60
    // hi 2^32 = (hi >> 29) 2^61 + (hi mod 2^29) 2^32 = (hi >> 29) + (hi mod 2^29) 2^32
    const long long tot = lo + (hi >> 29) + (long long)(((u64)hi & ((1ULL << 29) - 1)) << 32) + (long long)(2 * SS_P);
    return ss_reduce((u64)tot + more);   // 2^61 < tot < 2^63
}
#endif

}  // namespace SS_NS
