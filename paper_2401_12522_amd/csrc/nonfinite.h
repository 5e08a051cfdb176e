// A product P V under a mask has to leave out what the mask leaves out, also where it is no number: a matrix instruction gives
// 0 * inf = NaN for a masked key's infinity.  Where a tile that the mask cuts holds infinities or NaN in V (looked for there alone), they are taken
// out of the product, and three products of zeros and ones say where they belong.
#pragma once
#include "common.h"

// bit 15 of every half of w that is an infinity or a NaN in bf16
__device__ __forceinline__ uint32_t nonfinite_halves(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ bool has_nonfinite(bf16x8 v) {
    const uint4 u = __builtin_bit_cast(uint4, v);
    return (nonfinite_halves(u.x) | nonfinite_halves(u.y) | nonfinite_halves(u.z) | nonfinite_halves(u.w)) != 0;
}
// the larger magnitude bits of each half of m and of all pairs of v
__device__ __forceinline__ uint32_t largest_halves(uint32_t m, bf16x8 v) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u4;
    typedef __attribute__((ext_vector_type(2))) unsigned short h2;
    const u4 x = __builtin_bit_cast(u4, v);
#pragma unroll
    for (int i = 0; i < 4; i++) m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(h2, m), __builtin_bit_cast(h2, x[i] & 0x7FFF7FFFu)));
    return m;
}
// v without its infinities and NaN; not 0 if there were any
__device__ __forceinline__ uint32_t drop_nonfinite(bf16x8 &v) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u4;
    u4 x = __builtin_bit_cast(u4, v);
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t bad = nonfinite_halves(x[i]);
        x[i] &= ~((bad >> 15) * 0xFFFFu);
        any |= bad;
    }
    v = __builtin_bit_cast(bf16x8, x);
    return any;
}
// v without its infinities and NaN; up: 1 where v is +inf or NaN; down: 1 where it is -inf or NaN.  (Two halves a word at a time: compares of
// single values would take a pair of scalar registers each.)
__device__ __forceinline__ void split_nonfinite(bf16x8 &v, bf16x8 &up, bf16x8 &down) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u4;
    u4 x = __builtin_bit_cast(u4, v), a, b;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t w = x[i], bad = nonfinite_halves(w), nan = ((((w & 0x007F007Fu) + 0x007F007Fu) & 0x00800080u) << 8) & bad;
        a[i] = ((nan | (bad & ~w)) >> 15 & 0x00010001u) * 0x3F80u;
        b[i] = ((nan | (bad & w)) >> 15 & 0x00010001u) * 0x3F80u;
        x[i] = w & ~((bad >> 15) * 0xFFFFu);
    }
    v = __builtin_bit_cast(bf16x8, x);
    up = __builtin_bit_cast(bf16x8, a);
    down = __builtin_bit_cast(bf16x8, b);
}
// What a count of visible infinities adds to a sum (a NaN is both +inf and -inf, which together are one): 0 or an infinity.  (Not by a product:
// fused with the sum it would stay finite.)
__device__ __forceinline__ float nonfinite_term(float count) { return ldexpf(count, 255); }
