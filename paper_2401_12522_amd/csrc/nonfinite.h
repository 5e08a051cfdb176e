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
// v without its infinities and NaN; up: 1 where v is +inf or NaN; down: 1 where it is -inf or NaN
__device__ __forceinline__ void split_nonfinite(bf16x8 &v, bf16x8 &up, bf16x8 &down) {
    typedef __attribute__((ext_vector_type(8))) uint16_t u8;
    u8 x = __builtin_bit_cast(u8, v), a, b;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const bool bad = (x[e] & 0x7F80) == 0x7F80, nan = bad && (x[e] & 0x7F);
        a[e] = bad && (nan || !(x[e] & 0x8000)) ? 0x3F80 : 0;
        b[e] = bad && (nan || (x[e] & 0x8000)) ? 0x3F80 : 0;
        x[e] = bad ? 0 : x[e];
    }
    v = __builtin_bit_cast(bf16x8, x);
    up = __builtin_bit_cast(bf16x8, a);
    down = __builtin_bit_cast(bf16x8, b);
}
// what the counts of visible +inf and -inf (a NaN is both) add to a sum
__device__ __forceinline__ float nonfinite_term(float up, float down) { return (up > 0.f ? INFINITY : 0.f) + (down > 0.f ? -INFINITY : 0.f); }
