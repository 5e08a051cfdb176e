// Microscaled blocks of the 4- and 8-bit K/V cache (bita_kv_mx) on the device: where a slot's row lies, and blocks to and from bf16.
#pragma once
#include "common.h"

struct KvMx {
    unsigned char *k, *v;
    uint8_t *k_scale, *v_scale;
    const int32_t *table;               // nullptr: contiguous, a sequence a page
    int batch, Hkv, smax, page_lg, page_rows, slot_mask, n_pages, max_pages;
};

// Row of slot j of (sequence, head): codes at row * HD * BITS / 8, scales at row * HD / 32.
__device__ __forceinline__ int64_t mx_row(const KvMx &kv, int b, int h, int j) {
    const int page = kv.table ? min(max(kv.table[(int64_t)b * kv.max_pages + (j >> kv.page_lg)], 0), kv.n_pages - 1) : b;
    return ((int64_t)page * kv.Hkv + h) * kv.page_rows + (j & kv.slot_mask);
}

// The scale byte of a block whose largest magnitude has these fp32 bits (NaN and infinity: 255, as integers they are above the rest).
// 4 bits: the largest code is 6, and what is below 7 rounds to it: a < 7 2^e.  With a = (1 + m) 2^(E - 127) that is e = E - 129 where
// 1 + m < 1.75, else one more.  8 bits: 448, and what is up to 464 (a tie, to the even 448): e = E - 135 where 1 + m <= 1.8125.
template <int BITS>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
    const int E = (int)(top >> 23);
    const uint32_t m = top & 0x7FFFFFu;
    if (E == 255) return 255;
    return BITS == 4 ? max(E - 2 + (m >= 0x600000u ? 1 : 0), 2) : max(E - 8 + (m > 0x680000u ? 1 : 0), 10);
}
// 2^e of a scale byte; NaN for 255 (a conversion with it gives NaN)
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte == 255 ? 0x7FC00000u : byte << 23); }

typedef __attribute__((ext_vector_type(2))) __bf16 mx_bf16x2;
typedef __attribute__((ext_vector_type(2))) float mx_f32x2;
typedef __attribute__((ext_vector_type(2))) short mx_s16x2;

// eight values to codes: one dword of 4-bit codes, two of 8-bit ones (the conversions divide by the scale and round to nearest even, once)
__device__ __forceinline__ uint32_t mx_encode4(const float (&v)[8], float scale) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
    return r;
}
__device__ __forceinline__ uint2 mx_encode8(const float (&v)[8], float scale) {
    mx_s16x2 a = {0, 0}, b = {0, 0};
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, v[0], v[1], scale, false);
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, v[2], v[3], scale, true);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, v[4], v[5], scale, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, v[6], v[7], scale, true);
    return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}
// eight codes to bf16 (exact)
__device__ __forceinline__ bf16x8 mx_decode4(uint32_t c, float scale) {
    mx_bf16x2 p[4];
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
    return bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}
__device__ __forceinline__ bf16x8 mx_decode8(uint32_t lo, uint32_t hi, float scale) {
    mx_bf16x2 p[4];
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}

// where row r of head h of sequence b lies in a tensor of rows (elements)
struct MxRows {
    int64_t seq, head, row;
    __host__ __device__ __forceinline__ int64_t at(int b, int h, int r) const { return b * seq + h * head + r * row; }
};
// host: strides as given, those of axes with one place (which are nobody's) as 0
inline MxRows mx_rows(int64_t seqs, int64_t seq, int64_t heads, int64_t head, int64_t rows, int64_t row) {
    return MxRows{seqs > 1 ? seq : 0, heads > 1 ? head : 0, rows > 1 ? row : 0};
}

// host: strides and pointers as the kernels' 16-byte accesses need them
int mx_rows_check(const char *who, const MxRows &k, const MxRows &v, uintptr_t pointers);
// host: the descriptor checked and as the kernels take it (kv_mx.hip)
int kv_mx_of(const bita_kv_mx *kv, KvMx *out, const char *who);
