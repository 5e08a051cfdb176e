// The inner part of attention for many queries: a wave holds 32 queries of a head and their running softmax, and takes tiles of 64 keys whose
// K and V rows lie in LDS as bf16.
//  * S^T = K Q^T and O^T = V^T P^T by 32 x 32 x 16 matrix instructions.  Lane (h, c) = (l / 32, l % 32) has the scores of query c for keys
//    8 i + 4 h + 0..3 of each half of the tile, which is the B operand of the second product if that takes the keys in this
//    order: the probabilities stay in registers, and a maximum or a sum crosses lanes once.
//  * K rows are read by 16-byte columns, V rows by transposed reads (four keys of 16 columns a group of 16 lanes).  Both are swizzled, so that
//    neighbouring rows lie in different banks: column p of row r is at p ^ swizzle(r).
//  * The transposed reads are bare instructions: next tiles reach LDS by loads that the kernels track themselves, and the compiler,
//    which cannot tell the buffers apart, would drain those before each such read.  Their results are valid behind the wait that
//    takes the registers through itself.
#pragma once
#include "nonfinite.h"
#include <type_traits>

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;

#define CORE_KEYS 64
#define CORE_SUM 0x1p24f                // the largest sum of a lane's 32 probabilities of a tile that leaves their reference where it is (of a true maximum: 2^5)
#define CORE_FAR 0x1p23f                // the largest maximum (of products, before their scaling) whose scaled value is a reference good to an eighth of an octave

__device__ __forceinline__ float core_exp2(float x) { return __builtin_amdgcn_exp2f(x); }       // results below 2^-126 are zero
__device__ __forceinline__ uint32_t core_pk_bf16(float a, float b) {
    typedef __attribute__((ext_vector_type(2))) float f2;
    typedef __attribute__((ext_vector_type(2))) __bf16 b2;
    const f2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
}
__device__ __forceinline__ float core_max_halves(float x) {
    typedef __attribute__((ext_vector_type(2))) unsigned u2;
    const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float core_sum_halves(float x) {
    typedef __attribute__((ext_vector_type(2))) unsigned u2;
    const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int OFFSET>
__device__ __forceinline__ s16x4_t core_read_tr(uint32_t addr) {
    static_assert(OFFSET >= 0 && OFFSET < 65536, "ds offset field");
    s16x4_t v;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFFSET));
    return v;
}
template <int OFFSET>
__device__ __forceinline__ u32x4_t core_read_b128(uint32_t addr) {
    static_assert(OFFSET >= 0 && OFFSET < 65536, "ds offset field");
    u32x4_t v;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFFSET));
    return v;
}
// this lane's number, worked out where it is asked for: kept through a loop it takes a register
__device__ __forceinline__ int core_lane() {
    int l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(l));
    return l;
}
template <int I, int N, typename F>
__device__ __forceinline__ void core_for(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        core_for<I + 1, N>(f);
    }
}

template <int HD>
struct AttnCore {
    static constexpr int KS = HD / 16, NT = HD / 32, ROW = HD * 2, TILE = CORE_KEYS * ROW;
    bf16x8 q[KS];                       // lane (h, c), k-step s: query c, values 16 s + 8 h ..
    f32x16 o[NT];                       // lane (h, c), tile n, register 4 i + r: query c, column 32 n + 8 i + 4 h + r
    float m_run, l_run, base;           // the largest score, this lane's part of the sum of 2^(score scale - base)
    uint32_t k_at, v_at[2];             // this lane's place in a K tile, in a V tile (keys 8 x + 4 h .. of a 16, x = 0, 1)

    static __device__ __forceinline__ int k_swizzle(int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; }
    static __device__ __forceinline__ int v_swizzle(int r) { return (HD == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1)) + ((r >> 2) & 3); }

    __device__ __forceinline__ void init(int lane) {
        const int h = lane >> 5, c = lane & 31;
#pragma unroll
        for (int n = 0; n < NT; n++) o[n] = f32x16{};
        m_run = -INFINITY;
        l_run = base = 0.f;
        k_at = c * ROW + ((h ^ k_swizzle(c)) * 16);
#pragma unroll
        for (int x = 0; x < 2; x++) {
            const int r = 8 * x + 4 * h + ((c & 15) >> 2), col = (c & 16) + 4 * (c & 3);
            v_at[x] = r * ROW + (((col >> 3) ^ v_swizzle(r)) * 16) + (col & 4) * 2;
        }
    }
    // K fragments of four k-steps (k-steps sit in address bits that the swizzle shares by exclusive or), two groups of them in flight
    struct KFrag { u32x4_t f[4]; };
    template <int G>
    __device__ __forceinline__ void k_read(uint32_t at, KFrag &k) const {
        core_for<0, 4>([&](auto i_) __attribute__((always_inline)) {
            constexpr int step = (4 * G + decltype(i_)::value) % KS, h = (4 * G) / KS;
            k.f[decltype(i_)::value] = core_read_b128<h * 32 * ROW>(at ^ (32 * step));
        });
    }
    template <int N>
    static __device__ __forceinline__ void k_wait(KFrag &k) {
        asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(k.f[0]), "+v"(k.f[1]), "+v"(k.f[2]), "+v"(k.f[3]) : "n"(N));
    }
    __device__ __forceinline__ void scores(uint32_t tile, f32x16 (&s)[2]) const {
        constexpr int GROUPS = 2 * KS / 4;
        const uint32_t at = tile + k_at;
        KFrag k[2];
        k_read<0>(at, k[0]);
        core_for<0, GROUPS>([&](auto g_) __attribute__((always_inline)) {
            constexpr int g = decltype(g_)::value, h = 4 * g / KS;
            if constexpr (g + 1 < GROUPS) k_read<g + 1>(at, k[(g + 1) & 1]);
            k_wait<(g + 1 < GROUPS) ? 4 : 0>(k[g & 1]);
            if constexpr (4 * g % KS == 0) s[h] = f32x16{};
#pragma unroll
            for (int i = 0; i < 4; i++)
                s[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[g & 1].f[i]), q[(4 * g + i) % KS], s[h], 0, 0, 0);
        });
    }
    static __device__ __forceinline__ float largest(const f32x16 (&s)[2]) {
        float m = fmaxf(s[0][0], s[1][0]);
#pragma unroll
        for (int e = 1; e < 16; e++) m = fmaxf(m, fmaxf(s[0][e], s[1][e]));
        return m;
    }
    // the running maximum takes the next tile's in; it moves rarely after the first tiles, and only then are sums rescaled
    __device__ __forceinline__ void take_maximum(float mx, float scale_log2) {
        if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
            const float m_new = fmaxf(m_run, core_max_halves(mx));
            // in two halves: what is rescaled may be far above 1, and one factor below 2^-126 would be 0
            const float alpha = m_new == -INFINITY ? 1.f : core_exp2((m_run - m_new) * (0.5f * scale_log2));
            m_run = m_new;
            base = m_new == -INFINITY ? 0.f : m_new * scale_log2;
            l_run = l_run * alpha * alpha;
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int e = 0; e < 16; e++) o[n][e] = o[n][e] * alpha * alpha;
        }
    }
    // scores to probabilities 2^(score scale - base) as bf16 pairs, in the order of the registers; their sum, taken before they are rounded (rounded to
    // bf16 a probability is off by at most 2^-8 of itself, as the result is; the sum of the rounded ones, by the pairs' dot product, brought the error at 8192
    // tokens from 0.0022 to 0.0020 of the result, 0.0016 of which is the result's own rounding, for 2 % of the time)
    // (The maximum is taken off before the scaling here, so that it has weight 1 however large it is; `base` is that to its own rounding.)
    __device__ __forceinline__ float exponentials(const f32x16 (&s)[2], float scale_log2, uint32_t (&p)[16]) const {
        const float top = m_run == -INFINITY ? 0.f : m_run;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float a = core_exp2((s[e >> 4][e & 15] - top) * scale_log2), b = core_exp2((s[e >> 4][(e & 15) + 1] - top) * scale_log2);
            sum[0] += a;
            sum[1] += b;
            p[e >> 1] = core_pk_bf16(a, b);
        }
        return sum[0] + sum[1];
    }
    // The reference `base` need not be the maximum: bf16 and fp32 have one range of exponents, so a probability above 1 loses nothing by itself, and the tile's
    // maximum is looked for (look) only before a sum passes CORE_SUM, while there is no maximum (a query whose scores were all -inf has no reference, and what
    // it summed without one would be dropped with the first that it gets), or where it is so large that the reference's rounding is octaves.  (Nothing above 2^-126
    // of the largest is lost.)
    // The products with V share that range: n keys have a sum of up to 2^19 n, so values are finite on the way up to max |v| = 2^108 / n (with the true maximum, 2^127 / n).  What the limit
    // costs where scores spread widely, by 1, 3 and 10 nats: 8192 tokens 982, 1002, 1070 us, four trees of 68 rows 54, 52.4, 61; with 2^16 983, 1015, 1097 and 54, 53.3, 66, with 2^6
    // 1004, 1096, 1180 and 55, 63, 70; with 2^60, where values of 2^68 overflowed, 984, 1001, 1006 and 54, 52.5, 53.
    __device__ __forceinline__ void probabilities(f32x16 (&s)[2], float scale_log2, uint32_t (&p)[16], bool look) {
        float sum;
        for (;;) {
            if (look) {
                asm volatile("" : "+v"(s[0]), "+v"(s[1]));                      // (else the maximum is taken of every tile, ahead of time)
                take_maximum(largest(s), scale_log2);
            }
            sum = exponentials(s, scale_log2, p);
            if (look || __builtin_amdgcn_ballot_w64(sum > CORE_SUM || !(fabsf(m_run) < CORE_FAR)) == 0) break;
            look = true;
        }
        l_run += sum;
    }
    // The next tile's scores while this one's become probabilities: the matrix instructions of the first between the vector instructions of the
    // second, pair by pair.
    __device__ __forceinline__ void scores_and_probabilities(uint32_t tile, f32x16 (&next)[2], f32x16 (&s)[2], float scale_log2, uint32_t (&p)[16]) {
        constexpr int GROUPS = 2 * KS / 4, PAIRS = 16 / (2 * KS);               // pairs of probabilities behind each matrix instruction
        uint32_t at = tile + k_at;
        asm volatile("" : "+v"(at));                                            // (what follows from it is worked out here: kept for both tiles of a pair it takes registers)
        KFrag k[2];
        float sum[2] = {0.f, 0.f};
        __builtin_amdgcn_s_setprio(1);                                          // (ahead of the other wave's single products: 8192 tokens 1087 -> 1067 us)
        k_read<0>(at, k[0]);
        core_for<0, GROUPS>([&](auto g_) __attribute__((always_inline)) {
            constexpr int g = decltype(g_)::value, h = 4 * g / KS;
            if constexpr (g + 1 < GROUPS) k_read<g + 1>(at, k[(g + 1) & 1]);
            k_wait<(g + 1 < GROUPS) ? 4 : 0>(k[g & 1]);
            if constexpr (4 * g % KS == 0) next[h] = f32x16{};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                next[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[g & 1].f[i]), q[(4 * g + i) % KS], next[h], 0, 0, 0);
#pragma unroll
                for (int j = 0; j < PAIRS; j++) {
                    const int e = 2 * ((4 * g + i) * PAIRS + j);
                    const float x = core_exp2(__builtin_fmaf(s[e >> 4][e & 15], scale_log2, -base)), y = core_exp2(__builtin_fmaf(s[e >> 4][(e & 15) + 1], scale_log2, -base));
                    sum[0] += x;
                    sum[1] += y;
                    p[e >> 1] = core_pk_bf16(x, y);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        });
        __builtin_amdgcn_s_setprio(0);
        float total = sum[0] + sum[1];
        if (__builtin_amdgcn_ballot_w64(total > CORE_SUM || !(fabsf(m_run) < CORE_FAR)) != 0) {
            asm volatile("" : "+v"(s[0]), "+v"(s[1]));                          // (else the maximum is taken of every tile, ahead of time)
            take_maximum(largest(s), scale_log2);
            total = exponentials(s, scale_log2, p);
        }
        l_run += total;
    }
    // V fragments of 16 keys: column tile n of the head
    struct VFrag { s16x4_t half[NT][2]; };
    template <int KK>
    __device__ __forceinline__ void v_read(const uint32_t (&at)[2], VFrag &v) const {
#pragma unroll
        for (int n = 0; n < NT; n++) {
            v.half[n][0] = core_read_tr<16 * KK * ROW>(at[0] ^ (64 * n));
            v.half[n][1] = core_read_tr<16 * KK * ROW>(at[1] ^ (64 * n));
        }
    }
    // at most N of the wave's LDS operations are outstanding: these fragments are there
    template <int N>
    static __device__ __forceinline__ void v_wait(VFrag &v) {
        if constexpr (NT == 4)
            asm volatile("s_waitcnt lgkmcnt(%8)" : "+v"(v.half[0][0]), "+v"(v.half[0][1]), "+v"(v.half[1][0]), "+v"(v.half[1][1]), "+v"(v.half[2][0]),
                         "+v"(v.half[2][1]), "+v"(v.half[3][0]), "+v"(v.half[3][1]) : "n"(N));
        else
            asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(v.half[0][0]), "+v"(v.half[0][1]), "+v"(v.half[1][0]), "+v"(v.half[1][1]) : "n"(N));
    }
    static __device__ __forceinline__ bf16x8 v_fragment(const VFrag &v, int n) {
        typedef __attribute__((ext_vector_type(8))) short s8;
        return __builtin_bit_cast(bf16x8, s8{v.half[n][0][0], v.half[n][0][1], v.half[n][0][2], v.half[n][0][3], v.half[n][1][0], v.half[n][1][1], v.half[n][1][2], v.half[n][1][3]});
    }
    static __device__ __forceinline__ bf16x8 p_fragment(const uint32_t (&p)[16], int kk) {
        return __builtin_bit_cast(bf16x8, make_uint4(p[4 * kk], p[4 * kk + 1], p[4 * kk + 2], p[4 * kk + 3]));
    }
    // o += V^T P^T of a tile.  MASKED: without V's infinities and NaN; whether there were any is noted in `odd`, and add_nonfinite
    // puts them where they are seen once everything else is done.  (They are looked for by the largest magnitude of 16 keys, two instructions a pair of values.)
    template <bool MASKED>
    __device__ __forceinline__ void add_values(uint32_t tile, const uint32_t (&p)[16], uint32_t &odd) {
        uint32_t at[2] = {tile + v_at[0], tile + v_at[1]};
        asm volatile("" : "+v"(at[0]), "+v"(at[1]));
        VFrag v[2];
        v_read<0>(at, v[0]);
        core_for<0, CORE_KEYS / 16>([&](auto kk_) __attribute__((always_inline)) {
            constexpr int kk = decltype(kk_)::value;
            if constexpr (kk + 1 < CORE_KEYS / 16) v_read<kk + 1>(at, v[(kk + 1) & 1]);
            v_wait<(kk + 1 < CORE_KEYS / 16) ? 2 * NT : 0>(v[kk & 1]);
            bf16x8 x[NT];
#pragma unroll
            for (int n = 0; n < NT; n++) x[n] = v_fragment(v[kk & 1], n);
            if constexpr (MASKED) {
                uint32_t top = 0;
#pragma unroll
                for (int n = 0; n < NT; n++) top = largest_halves(top, x[n]);
                if (__builtin_amdgcn_ballot_w64(nonfinite_halves(top) != 0) != 0) {
#pragma unroll
                    for (int n = 0; n < NT; n++) odd |= drop_nonfinite(x[n]);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; n++) o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[n], p_fragment(p, kk), o[n], 0, 0, 0);
        });
    }
    // This lane's query's result o * scale as bf16, at dst (of its row).  The half waves (h) trade eights of columns, so that a lane writes 16 bytes.
    __device__ __forceinline__ void put(uint16_t *dst, float scale, int h) const {
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                typedef __attribute__((ext_vector_type(2))) unsigned u2;
                const u2 a = __builtin_amdgcn_permlane32_swap(core_pk_bf16(o[n][4 * i] * scale, o[n][4 * i + 1] * scale),
                                                              core_pk_bf16(o[n][4 * i + 4] * scale, o[n][4 * i + 5] * scale), false, false);
                const u2 b = __builtin_amdgcn_permlane32_swap(core_pk_bf16(o[n][4 * i + 2] * scale, o[n][4 * i + 3] * scale),
                                                              core_pk_bf16(o[n][4 * i + 6] * scale, o[n][4 * i + 7] * scale), false, false);
                *reinterpret_cast<uint4 *>(dst + 32 * n + 8 * (i + h)) = make_uint4(a[0], b[0], a[1], b[1]);
            }
    }
    // The infinities and NaN of up to 64 rows of V (row r at v + r * ld, the last one's number is `last`), seen where `seen` has the key's bit for this
    // lane's query.  Rare, and slow: single values from memory.
    __device__ __forceinline__ void add_nonfinite(const uint16_t *v, int64_t ld, int last, uint64_t seen) {
        const int h = (threadIdx.x >> 5) & 1, c = threadIdx.x & 31;
#pragma unroll 1
        for (int kk = 0; kk < CORE_KEYS / 16; kk++) {
            uint32_t one[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const uint64_t b = seen >> (16 * kk + 8 * (e >> 1) + 4 * h + 2 * (e & 1));
                one[e] = (b & 1 ? 0x3F80u : 0u) | (b & 2 ? 0x3F800000u : 0u);
            }
            const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(one[0], one[1], one[2], one[3]));
#pragma unroll
            for (int n = 0; n < NT; n++) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int r = 16 * kk + 8 * (e >> 1) + 4 * h + 2 * (e & 1);
                    w[e] = v[min(r, last) * ld + 32 * n + c] | (uint32_t)v[min(r + 1, last) * ld + 32 * n + c] << 16;
                }
                bf16x8 x = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3])), up, down;
                split_nonfinite(x, up, down);
                f32x16 count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(up, ones, f32x16{}, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 16; e++) o[n][e] += nonfinite_term(count[e]);
                count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(down, ones, f32x16{}, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 16; e++) o[n][e] -= nonfinite_term(count[e]);
            }
        }
    }
};
