// Rows held as 8-bit integers with one fp32 scale each, and the kernels that produce them: RMSNorm with the residual's addition,
// SwiGLU gating, and plain rows (attention outputs, weights).  A row v is held as
//     q_i = round(127 v_i / a),  ties to even,  s = a / 127,  a = max |v_i|        (a = 0: q = 0, s = 0)
// so that v_i is q_i s within half a step.  A row with a NaN or an infinity has q = 0 and s = NaN: every product of it is NaN.
//
// Which side of a rounding border a value falls on is decided exactly for the norm and for plain rows, and in double for the
// gating: two programs that agree on the inputs agree on every q.  A code is found in fp32 (relative error of 127 |v| / a below
// 1e-6) and, where that lands too near to a border, again in double.  The norm's row factor r > 0 scales v and a alike
// and drops out of q, so that v stands for h_i g_i, which a double holds exactly (24 + 8 bits); whether |v| is above, on or below
// the border (k + 1/2) a / 127 is whether 254 |v| - (2k + 1) a is positive, zero or negative, both terms exact in a double.
//
// One workgroup per row, whose values v it holds in registers as fp32: one pass over memory, one barrier for the row's maximum and sum
// (the norm's and the gating's maximum is refined in double behind a second one: by the few threads that hold a candidate, who read
// its sources again; held in registers they made the few rows no faster and the gating spill).  What bounds it is memory where there
// are many rows, provided that a value costs few instructions and a row few waits: values in groups of eight a thread, one branch a
// group for all that is rare (34, 26 and 16 vector instructions a value for norm, gating and plain rows, bf16), the waves' maxima and
// sums read side by side (one after the other they cost more than the row: 11008 rows of 4096 bf16 91 us).
#include "common.h"

enum { ROWS_PLAIN = 0, ROWS_NORM = 1, ROWS_GATE = 2 };

// fp32 quotients 127 |v| / a are found again in double where they are this near to a border: 127 times their relative error, in units
// of 2^-24: 127 / a at most 2 and its product with v 1, for plain rows no more (2.3e-5); the norm's v and a, products, 1 each (3.8e-5); the
// gating's v and a 8 each (exponential 2 and its correction 1, sum 1, reciprocal 2, two products; 1.44e-4).
template <int KIND>
constexpr float round_margin() { return KIND == 0 ? 2.5e-5f : KIND == 1 ? 4.0e-5f : 1.5e-4f; }
// largest |v| of a row for which fp32 quotients have that error: 127 / a and all that matters are normal numbers
#define PLAIN_RANGE_LO 1e-30f
#define PLAIN_RANGE_HI 1e30f
// gates below this are taken in double: exp(-gate) nears the end of fp32
#define GATE_LOW -80.0f
// rows from which on four waves take a row
#define ROWS_MANY 1024

struct RowsArgs {
    const void *x, *delta;            // ROWS_GATE: x holds gate and up columns
    const uint16_t *gain;             // ROWS_NORM: bf16 [k]
    void *total;                      // ROWS_NORM: x + delta (may be x)
    int8_t *q;
    float *scale;
    int64_t ldx, ld_delta, ld_total, ldq;
    SumsQ8 sums;                      // ROWS_NORM, SUMS: the delta (`delta` is sums.part)
    int64_t sums_step;                // from one split's to the next
    int k, tile;                      // ROWS_GATE: columns of a gate tile (its up tile follows), 16 or k
    double eps;
};

__device__ __forceinline__ uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }       // nearest even; a NaN stays one

// (16 and 8 bytes at an element's alignment: the hardware takes them)
struct __attribute__((packed, aligned(2))) Halves8 { uint32_t w[4]; };
struct __attribute__((packed, aligned(4))) Words8 { float v[8]; };
struct __attribute__((packed, aligned(1))) Bytes8 { uint32_t w[2]; };

// n values of a row from column `at`, 8 but for the row's last
template <bool BF16>
__device__ __forceinline__ void load8(const void *row, int at, int n, float v[8]) {
    if (n == 8) {
        if constexpr (BF16) {
            const Halves8 u = *reinterpret_cast<const Halves8 *>((const uint16_t *)row + at);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                v[2 * e] = __uint_as_float(u.w[e] << 16);
                v[2 * e + 1] = __uint_as_float(u.w[e] & 0xFFFF0000u);
            }
        } else {
            const Words8 u = *reinterpret_cast<const Words8 *>((const float *)row + at);
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = u.v[e];
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        if constexpr (BF16) v[e] = e < n ? bf16_to_f32(((const uint16_t *)row)[at + e]) : 0.f;
        else v[e] = e < n ? ((const float *)row)[at + e] : 0.f;
    }
}
template <bool BF16>
__device__ __forceinline__ void store8(void *row, int at, int n, const float v[8]) {
    if (n == 8) {
        if constexpr (BF16) {
            Halves8 u;
#pragma unroll
            for (int e = 0; e < 4; e++) u.w[e] = (uint32_t)to_bf16(v[2 * e]) | ((uint32_t)to_bf16(v[2 * e + 1]) << 16);
            *reinterpret_cast<Halves8 *>((uint16_t *)row + at) = u;
        } else {
            Words8 u;
#pragma unroll
            for (int e = 0; e < 8; e++) u.v[e] = v[e];
            *reinterpret_cast<Words8 *>((float *)row + at) = u;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (e < n) {
            if constexpr (BF16) ((uint16_t *)row)[at + e] = to_bf16(v[e]);
            else ((float *)row)[at + e] = v[e];
        }
}

// silu(g) u = g u / (1 + exp(-g)) for g >= GATE_LOW: -g log2(e) in two words, so that the power of two is off by its own unit only.  Of a gate above
// 2.36e38 the first word is an infinity and this no number: its row is then taken in double as a whole (a gate limited for the exponent costs every
// value an instruction).  u is multiplied first: half of a subnormal gate would be rounded to a multiple of the smallest number, and a large u
// bring that error back; where u / (1 + exp(-g)) is rounded so, v is below 100 * 2^-126, and the rows that fp32 decides have a largest value of 1e-30 or more.
__device__ __forceinline__ float gated(float g, float u) {
    const float h = -g * 1.44269504f, l = __builtin_fmaf(-g, 1.92596303e-8f, __builtin_fmaf(-g, 1.44269504f, -h));
    const float p = __builtin_amdgcn_exp2f(h), e = __builtin_fmaf(p, l * 0.693147181f, p);
    return u * __builtin_amdgcn_rcpf(1.0f + e) * g;
}
__device__ __forceinline__ double gated_exactly(float g, float u) { return (double)g / (1.0 + exp(-(double)g)) * (double)u; }

// Maximum and sum over a wave or its first 16 lanes, the same in every lane: moves between lanes inside the vector unit (zero from
// outside: the values are >= 0), four shifts within 16 lanes and for a wave two broadcasts of 16 lanes' last, then one lane is read.
// Moves through LDS cost more: 68 plain rows of 4096 bf16 4.0 us (these: 3.65), norm of 68 rows of 8192 fp32 8.0 (7.4), 68 gated rows of
// 11008 fp32 8.0 (7.6), 11008 plain rows of 4096 bf16 29.5 (28.1).
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false); }
template <int CTRL>
__device__ __forceinline__ double moved(double v) {
    const uint64_t w = (uint64_t)__double_as_longlong(v);
    return __longlong_as_double((long long)((uint64_t)moved<CTRL>((uint32_t)(w >> 32)) << 32 | moved<CTRL>((uint32_t)w)));
}
__device__ __forceinline__ uint32_t lane_value(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ double lane_value(double v, int lane) {
    const uint64_t w = (uint64_t)__double_as_longlong(v);
    return __longlong_as_double((long long)((uint64_t)lane_value((uint32_t)(w >> 32), lane) << 32 | lane_value((uint32_t)w, lane)));
}
template <bool WAVE, bool SUM, typename T>
__device__ __forceinline__ T reduced(T v) {
#define ROWS_STEP(CTRL) { const T o = moved<CTRL>(v); if constexpr (SUM) v += o; else v = max(v, o); }
    ROWS_STEP(0x111) ROWS_STEP(0x112) ROWS_STEP(0x114) ROWS_STEP(0x118)               // row_shr 1, 2, 4, 8
    if constexpr (WAVE) { ROWS_STEP(0x142) ROWS_STEP(0x143) }                         // row_bcast 15, 31
#undef ROWS_STEP
    return lane_value(v, WAVE ? 63 : 15);
}

// fp32 + ROUNDER rounds to the nearest integer, ties to even, and has it (two's complement) in its low byte
#define ROUNDER 12582912.0f

// The delta's type where it is the sums of a product
#define SUMS 2
// eight neighbouring ones, as the product itself would store them in fp32: both products are rounded by themselves, wherever the compiler puts the
// addition that follows
__device__ __forceinline__ void load8_of_sums(const RowsArgs &a, int row, int at, float row_scale, float v[8]) {
#pragma clang fp contract(off)
    typedef __attribute__((ext_vector_type(4))) int i32x4;
    const int *part = a.sums.part + (int64_t)row * a.k + at;
    i32x4 sum[2] = {};
    for (int s0 = 0; s0 < a.sums.splits; s0 += 4) {
        i32x4 q[4][2];
#pragma unroll
        for (int s = 0; s < 4; s++)                          // (requested together; those past the last are left out)
#pragma unroll
            for (int e = 0; e < 2; e++) q[s][e] = reinterpret_cast<const i32x4 *>(part + min(s0 + s, a.sums.splits - 1) * a.sums_step)[e];
#pragma unroll
        for (int s = 0; s < 4; s++)
#pragma unroll
            for (int e = 0; e < 2; e++)
                if (s0 + s < a.sums.splits) sum[e] += q[s][e];
    }
    const float *scale = a.sums.col_scale + at;
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (float)sum[e >> 2][e & 3] * row_scale * scale[e];
}

// NV groups of 8 values per thread are held in registers.  KEEP false (rows longer than a workgroup holds; not the norm): the
// groups go round and the row is read again, mostly from cache.
template <int KIND, bool XB, int DT, int NV, bool KEEP>
__global__ __launch_bounds__(1024) void rows_q8_kernel(RowsArgs a) {
    static_assert(KEEP || KIND != ROWS_NORM, "the norm holds its row");
    __shared__ uint32_t s_max[16];
    __shared__ double s_sum[16];
    __shared__ unsigned long long s_exact;
    constexpr unsigned long long NO_NUMBER = ~0ull, BEYOND_FP32 = 0x47EFFFFFF0000000ull;      // (the latter 2^128 - 2^103, which rounds to an infinity)
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6, k = a.k;
    const char *x = (const char *)a.x + (int64_t)row * a.ldx * (XB ? 2 : 4);
    int8_t *q = a.q + (int64_t)row * a.ldq;
    float h[NV][8];                                         // the row's values; ROWS_NORM: h g

    // (ROWS_GATE) the gate column of value `at`; its up column is a.tile further
    auto gate_column = [&](int at) __attribute__((always_inline)) { return a.tile == 16 ? ((at >> 4) << 5) + (at & 15) : at; };
    auto one = [&](const void *p, int at) __attribute__((always_inline)) { return XB ? bf16_to_f32(((const uint16_t *)p)[at]) : ((const float *)p)[at]; };
    // value `at` in double, from memory (ROWS_NORM: from what this thread stored there)
    auto exactly = [&](int at) __attribute__((always_inline)) {
        if constexpr (KIND == ROWS_GATE) {
            const int col = gate_column(at);
            return gated_exactly(one(x, col), one(x, col + a.tile));
        } else if constexpr (KIND == ROWS_PLAIN) {
            return (double)one(x, at);
        } else {
            const float v = one(a.delta ? (const char *)a.total + (int64_t)row * a.ld_total * (XB ? 2 : 4) : x, at), g = bf16_to_f32(a.gain[at]);
            const uint32_t bits = max(__float_as_uint(v) & 0x7FFFFFFFu, __float_as_uint(g) & 0x7FFFFFFFu);
            return bits >= 0x7F800000u ? __longlong_as_double((long long)NO_NUMBER) : (double)v * (double)g;
        }
    };
    auto column = [&](int turn, int v) __attribute__((always_inline)) { return ((turn * NV + v) * (int)blockDim.x + tid) * 8; };
    auto fetch = [&](int v, int at) __attribute__((always_inline)) {
        const int n = min(max(k - at, 0), 8);
        if (n <= 0) {
#pragma unroll
            for (int e = 0; e < 8; e++) h[v][e] = 0.f;
        } else if constexpr (KIND == ROWS_GATE) {
            float g[8], u[8];
            const int col = gate_column(at);
            load8<XB>(x, col, n, g);
            load8<XB>(x, col + a.tile, n, u);
            float least = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                h[v][e] = gated(g[e], u[e]);
                least = fminf(least, g[e]);
            }
            if (least < GATE_LOW) {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (g[e] < GATE_LOW) h[v][e] = (float)gated_exactly(g[e], u[e]);
            }
        } else {
            load8<XB>(x, at, n, h[v]);
        }
    };

    // |v| as bits: any infinity or NaN is above every number
    uint32_t top_bits = 0;
    double sum = 0.0;
    const int turns = KEEP ? 1 : (k + NV * (int)blockDim.x * 8 - 1) / (NV * (int)blockDim.x * 8);
    for (int turn = 0; turn < turns; turn++) {
#pragma unroll
        for (int v = 0; v < NV; v++) fetch(v, column(turn, v));
        if constexpr (KIND == ROWS_NORM) {
            float d[NV][8], g[NV][8];                        // (all of a thread's reads are asked for before any is used)
#pragma unroll
            for (int v = 0; v < NV; v++) {
                const int at = column(0, v), n = min(max(k - at, 0), 8);
                if (n > 0) load8<true>(a.gain, at, n, g[v]);
            }
            if (a.delta) {
                float row_scale = 0.f;
                if constexpr (DT == SUMS) row_scale = a.sums.row_scale[row];        // (may be `scale`, which is written behind the barriers)
#pragma unroll
                for (int v = 0; v < NV; v++) {
                    const int at = column(0, v), n = min(max(k - at, 0), 8);
                    if (n <= 0) continue;
                    if constexpr (DT == SUMS) load8_of_sums(a, row, at, row_scale, d[v]);
                    else load8<DT == BITA_BF16>((const char *)a.delta + (int64_t)row * a.ld_delta * (DT == BITA_BF16 ? 2 : 4), at, n, d[v]);
                }
            }
#pragma unroll
            for (int v = 0; v < NV; v++) {
                const int at = column(0, v), n = min(max(k - at, 0), 8);
                if (n <= 0) continue;
                if (a.delta) {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        h[v][e] += d[v][e];
                        if constexpr (XB) h[v][e] = bf16_to_f32(to_bf16(h[v][e]));         // (what is stored is what is normalised)
                    }
                    store8<XB>((char *)a.total + (int64_t)row * a.ld_total * (XB ? 2 : 4), at, n, h[v]);
                }
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const double hd = h[v][e];
                    sum = fma(hd, hd, sum);
                    h[v][e] *= g[v][e];
                }
            }
        }
#pragma unroll
        for (int v = 0; v < NV; v++)
#pragma unroll
            for (int e = 0; e < 8; e++) top_bits = max(top_bits, __float_as_uint(h[v][e]) & 0x7FFFFFFFu);
    }
    // the row's maximum (and sum of squares)
    const uint32_t mine_bits = top_bits;
    top_bits = reduced<true, false>(top_bits);
    if constexpr (KIND == ROWS_NORM) sum = reduced<true, true>(sum);
    if (lane == 0) {
        s_max[wave] = top_bits;
        if constexpr (KIND == ROWS_NORM) s_sum[wave] = sum;
    }
    if (KIND != ROWS_PLAIN && tid == 0) s_exact = 0;
    __syncthreads();
    {
        const bool some = (lane & 15) < waves;               // 16 lanes take a wave's result each
        top_bits = reduced<false, false>(some ? s_max[lane & 15] : 0u);
        if constexpr (KIND == ROWS_NORM) sum = reduced<false, true>(some ? s_sum[lane & 15] : 0.0);
    }
    bool bad = top_bits >= 0x7F800000u;
    const float top32 = __uint_as_float(top_bits);
    const bool in_range = top32 >= PLAIN_RANGE_LO && top32 <= PLAIN_RANGE_HI;
    if constexpr (KIND != ROWS_PLAIN) {
        // the largest value in double: of those that fp32 has within its error of its largest (all, where fp32 does not hold them; rows of zeros
        // among these, at a cost: 68 gated rows of 11008 fp32 7.2 us, with one of zeros 15.0, norm of 68 rows of 8192 6.9 and 10.7)
        const float near = in_range ? top32 * (1.0f - 1e-5f) : 0.f;
        if (!in_range || __uint_as_float(mine_bits) >= near) {
            unsigned long long best = 0;
            for (int turn = 0; turn < turns; turn++) {
                uint32_t todo = 0;
#pragma unroll
                for (int v = 0; v < NV; v++) {
                    const int at = column(turn, v);
                    if constexpr (!KEEP) fetch(v, at);
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        if (at + e < k && (!in_range || fabsf(h[v][e]) >= near)) todo |= 1u << (8 * v + e);
                }
                while (todo) {
                    const int i = __builtin_ctz(todo);
                    todo &= todo - 1;
                    const unsigned long long w = (unsigned long long)__double_as_longlong(exactly(column(turn, i >> 3) + (i & 7)));
                    best = max(best, w == NO_NUMBER ? w : w & ~(1ull << 63));
                }
            }
            if (best) atomicMax(&s_exact, best);
        }
    }
    // the codes that fp32 decides are stored, the others' bits are returned: all of a row that fp32 does not hold
    const float c32 = 127.0f / top32;
    auto round = [&](int turn) __attribute__((always_inline)) {
        uint32_t todo = 0;
#pragma unroll
        for (int v = 0; v < NV; v++) {
            const int at = column(turn, v);
            if constexpr (!KEEP) fetch(v, at);
            const int n = min(max(k - at, 0), 8);
            if (n <= 0) continue;
            if (!in_range) {
                todo |= (uint32_t)((1 << n) - 1) << (8 * v);
                continue;
            }
            float r[8], off = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float t = h[v][e] * c32;
                r[e] = t + ROUNDER;
                off = fmaxf(off, fabsf(t - (r[e] - ROUNDER)));
            }
            if (off > 0.5f - round_margin<KIND>()) {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (e < n && fabsf(h[v][e] * c32 - (r[e] - ROUNDER)) > 0.5f - round_margin<KIND>()) todo |= 1u << (8 * v + e);
            }
            uint32_t b[8];
#pragma unroll
            for (int e = 0; e < 8; e++) b[e] = __float_as_uint(r[e]);
            if (n == 8) {
                Bytes8 w;
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const uint32_t lo = __builtin_amdgcn_perm(b[4 * e + 1], b[4 * e], 0x0c0c0400), hi = __builtin_amdgcn_perm(b[4 * e + 3], b[4 * e + 2], 0x0c0c0400);
                    w.w[e] = lo | hi << 16;
                }
                *reinterpret_cast<Bytes8 *>(q + at) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (e < n) q[at + e] = (int8_t)(b[e] & 255);
            }
        }
        return todo;
    };
    uint32_t todo = 0;
    // (before the second barrier, while the few threads that refine the maximum wait for its sources: with narrower margins norm of 4096
    // rows of 16384 bf16 64.6 -> 59.7 us, 11008 plain rows of 4096 27.9 -> 27.1, gating within 1 %)
    if constexpr (KEEP) todo = round(0);
    double top = top32;
    if constexpr (KIND != ROWS_PLAIN) {
        __syncthreads();
        top = __longlong_as_double((long long)s_exact);
        if constexpr (KIND == ROWS_NORM) bad = s_exact == NO_NUMBER;
        // (fp32's own products may be on the other side of its end; their exact values, all taken in double there, are not)
        else bad = s_exact >= BEYOND_FP32;
    }
    const bool none = bad || top == 0.0;                     // (not in_range)
    if (tid == 0) {
        double s = top / 127.0;
        if constexpr (KIND == ROWS_NORM) s /= sqrt(sum / (double)k + a.eps);
        a.scale[row] = bad ? __builtin_nanf("") : top == 0.0 ? 0.f : (float)s;
    }
    for (int turn = 0; turn < turns; turn++) {
        if constexpr (!KEEP) todo = round(turn);
        if (none) {
#pragma unroll
            for (int v = 0; v < NV; v++) {
                const int at = column(turn, v), n = min(max(k - at, 0), 8);
                if (n == 8) *reinterpret_cast<Bytes8 *>(q + at) = Bytes8{};
                else
                    for (int e = 0; e < n; e++) q[at + e] = 0;
            }
            continue;
        }
        while (todo) {
            const int i = __builtin_ctz(todo), at = column(turn, i >> 3) + (i & 7);
            todo &= todo - 1;
            const double p = exactly(at), m = fabs(p);
            double up;
            if constexpr (KIND == ROWS_GATE) {
                up = rint(m * 127.0 / top);
            } else {
                const double low = floor(m * (127.0 / top)), over = fma(-(2.0 * low + 1.0), top, 254.0 * m);
                up = over > 0.0 || (over == 0.0 && ((int)low & 1)) ? low + 1.0 : low;
            }
            q[at] = (int8_t)(int)copysign(up, p);
        }
    }
}

// ---------------------------------------------------------------------------------------
#define ROWS_A_LAUNCH (1 << 21)        // (a grid has less than 2^32 threads)
template <int KIND, bool XB, int DT>
static void launch_rows(RowsArgs a, int m, hipStream_t s) {
    // Few rows: as many waves as there are groups, for a row is latency.  Many: four waves and several rows a CU, up to four groups a
    // thread for plain rows and two for the others, which compute more (four / two: 28672 plain rows of 8192 bf16 131 / 137 us; norm of
    // 8192 rows of 5120 bf16 96 / 78, of 8192 fp32 186 / 178; 4096 gated rows of 28672 bf16 170 / 162).
    constexpr int HELD = KIND == ROWS_PLAIN ? 4 : 2;
    const int groups = (a.k + 7) / 8, most = m >= ROWS_MANY ? 256 : 1024, needed = (groups + HELD - 1) / HELD;
    const int threads = max(min(most, (groups + 63) / 64 * 64), min(1024, (needed + 63) / 64 * 64)), nv = (groups + threads - 1) / threads;
    for (int left = m; left > 0; left -= ROWS_A_LAUNCH) {
        const dim3 grid(min(left, ROWS_A_LAUNCH));
#define ROWS_LAUNCH(NV, KEEP) hipLaunchKernelGGL((rows_q8_kernel<KIND, XB, DT, NV, KEEP>), grid, dim3(threads), 0, s, a)
        if (nv <= 1) ROWS_LAUNCH(1, true);
        else if (KIND == ROWS_NORM || nv <= 2) ROWS_LAUNCH(2, true);      // (1024 threads of two groups: the norm's longest row)
        else if constexpr (KIND != ROWS_NORM) {
            if (nv <= 4) ROWS_LAUNCH(4, true);
            else ROWS_LAUNCH(2, false);
        }
#undef ROWS_LAUNCH
        const int64_t done = ROWS_A_LAUNCH;
        a.x = (const char *)a.x + done * a.ldx * (XB ? 2 : 4);
        if (DT == SUMS) a.sums.part += done * a.k, a.sums.row_scale += done;
        else if (a.delta) a.delta = (const char *)a.delta + done * a.ld_delta * (DT == BITA_BF16 ? 2 : 4);
        if (a.delta) a.total = (char *)a.total + done * a.ld_total * (XB ? 2 : 4);
        a.q += done * a.ldq;
        a.scale += done;
    }
}

static bool type_ok(int32_t t) { return t == BITA_F32 || t == BITA_BF16; }
static bool at_element(const void *p, int32_t t) { return (uintptr_t)p % (t == BITA_BF16 ? 2 : 4) == 0; }

extern "C" int bita_quantize_rows(const void *d_x, int32_t x_type, int32_t m_rows, int64_t k, int64_t ldx, int8_t *d_q, int64_t ldq,
                                  float *d_scale, void *stream) {
    if (!d_x || !d_q || !d_scale || m_rows <= 0 || k <= 0 || !type_ok(x_type) || !at_element(d_x, x_type) || ldx < k || ldq < k)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_quantize_rows: bad argument");
    if (k > BITA_Q8_MAX_K) return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_quantize_rows: k %lld, at most %d", (long long)k, BITA_Q8_MAX_K);
    RowsArgs a = {};
    a.x = d_x; a.q = d_q; a.scale = d_scale; a.ldx = ldx; a.ldq = ldq; a.k = (int)k;
    if (x_type == BITA_BF16) launch_rows<ROWS_PLAIN, true, BITA_F32>(a, m_rows, (hipStream_t)stream);
    else launch_rows<ROWS_PLAIN, false, BITA_F32>(a, m_rows, (hipStream_t)stream);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}

extern "C" int bita_silu_mul_q8(const void *d_gate_up, int32_t x_type, int32_t m_rows, int64_t d_ffn, int64_t ldx, int32_t tile,
                                int8_t *d_q, int64_t ldq, float *d_scale, void *stream) {
    if (!d_gate_up || !d_q || !d_scale || m_rows <= 0 || d_ffn <= 0 || !type_ok(x_type) || !at_element(d_gate_up, x_type) ||
        ldx < 2 * d_ffn || ldq < d_ffn)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_silu_mul_q8: bad argument");
    if ((tile != 0 && tile != 16) || (tile == 16 && d_ffn % 16))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_silu_mul_q8: tile must be 0 (all gate columns first) or 16 (d_ffn a multiple of 16)");
    if (d_ffn > BITA_Q8_MAX_K) return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_silu_mul_q8: d_ffn %lld, at most %d", (long long)d_ffn, BITA_Q8_MAX_K);
    RowsArgs a = {};
    a.x = d_gate_up; a.q = d_q; a.scale = d_scale; a.ldx = ldx; a.ldq = ldq; a.k = (int)d_ffn; a.tile = tile ? tile : (int)d_ffn;
    if (x_type == BITA_BF16) launch_rows<ROWS_GATE, true, BITA_F32>(a, m_rows, (hipStream_t)stream);
    else launch_rows<ROWS_GATE, false, BITA_F32>(a, m_rows, (hipStream_t)stream);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}

extern "C" int bita_norm_q8(const void *d_x, int32_t x_type, int32_t m_rows, int64_t d, int64_t ldx, const void *d_delta,
                            int32_t delta_type, int64_t ld_delta, const void *d_gain, float eps, void *d_total, int64_t ld_total,
                            int8_t *d_q, int64_t ldq, float *d_scale, void *stream) {
    if (!d_x || !d_gain || !d_q || !d_scale || m_rows <= 0 || d <= 0 || !type_ok(x_type) || !at_element(d_x, x_type) ||
        !at_element(d_gain, BITA_BF16) || ldx < d || ldq < d || !(eps >= 0.f && eps <= 3.4e38f) ||
        (d_delta && (!type_ok(delta_type) || !at_element(d_delta, delta_type) || !at_element(d_total, x_type) || ld_delta < d || !d_total || ld_total < d)))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_norm_q8: bad argument");
    if (d > 1024 * RMS_MAX_CHUNKS)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_norm_q8: d %lld, at most %d", (long long)d, 1024 * RMS_MAX_CHUNKS);
    if (d_total == d_x && d_delta && m_rows > 1 && ld_total != ldx)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_norm_q8: d_total is d_x with another row stride");
    RowsArgs a = {};
    a.x = d_x; a.delta = d_delta; a.gain = (const uint16_t *)d_gain; a.total = d_total; a.q = d_q; a.scale = d_scale;
    a.ldx = ldx; a.ld_delta = ld_delta; a.ld_total = ld_total; a.ldq = ldq; a.k = (int)d; a.eps = (double)eps;
    hipStream_t s = (hipStream_t)stream;
    const bool db = d_delta && delta_type == BITA_BF16;
    if (x_type == BITA_BF16) {
        if (db) launch_rows<ROWS_NORM, true, BITA_BF16>(a, m_rows, s);
        else launch_rows<ROWS_NORM, true, BITA_F32>(a, m_rows, s);
    } else {
        if (db) launch_rows<ROWS_NORM, false, BITA_BF16>(a, m_rows, s);
        else launch_rows<ROWS_NORM, false, BITA_F32>(a, m_rows, s);
    }
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}

// x += the sums of a product (its d columns as many as x's, a multiple of 16), then as bita_norm_q8
int norm_q8_of_sums(float *d_x, int m_rows, int64_t d, const SumsQ8 &delta, const void *d_gain, float eps, int8_t *d_q, int64_t ldq, float *d_scale, hipStream_t s) {
    RowsArgs a = {};
    a.x = d_x; a.delta = delta.part; a.sums = delta; a.sums_step = (int64_t)m_rows * d; a.gain = (const uint16_t *)d_gain; a.total = d_x; a.q = d_q; a.scale = d_scale;
    a.ldx = a.ld_total = d; a.ldq = ldq; a.k = (int)d; a.eps = (double)eps;
    launch_rows<ROWS_NORM, false, SUMS>(a, m_rows, s);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}
