// Rows held as 8-bit integers with one fp32 scale each, and the kernels that produce them: RMSNorm with the residual's addition,
// SwiGLU gating, and plain rows (attention outputs, weights).  A row v is held as
//     q_i = round(127 v_i / a),  ties to even,  s = a / 127,  a = max |v_i|        (a = 0: q = 0, s = 0)
// so that v_i is q_i s within half a step.  A row with a NaN or an infinity has q = 0 and s = NaN: every product of it is NaN.
//
// Which side of a rounding border a value falls on is decided exactly for the norm and for plain rows, and in double for the
// gating: two programs that agree on the inputs agree on every q.  A code is found in fp32 (relative error of 127 |v| / a below
// 1e-6) and, where that lands within ROUND_MARGIN of a border, again in double.  The norm's row factor r > 0 scales v and a alike
// and drops out of q, so that v stands for h_i g_i, which a double holds exactly (24 + 8 bits); whether |v| is above, on or below
// the border (k + 1/2) a / 127 is whether 254 |v| - (2k + 1) a is positive, zero or negative, both terms exact in a double.
//
// One workgroup per row, which it holds in registers: one pass over memory, one barrier for the row's maximum and sum (the
// gating's maximum is refined in double behind a second one).
#include "common.h"

enum { ROWS_PLAIN = 0, ROWS_NORM = 1, ROWS_GATE = 2 };

// |fp32 quotient - border| below which a code is found again in double: 127 times the relative error of the fp32 quotient,
// which is at most 5 units of 2^-24 for the norm and plain rows, 8 for the gating (expf 1 ulp, sum, division, two products, the
// factor 127 / a and its product) = 6e-5
#define ROUND_MARGIN 1.0e-4f
// largest |v| of a row for which fp32 quotients have that error: 127 / a and all that matters are normal numbers
#define PLAIN_RANGE_LO 1e-30f
#define PLAIN_RANGE_HI 1e30f

struct RowsArgs {
    const void *x, *delta;            // ROWS_GATE: x holds gate and up columns
    const uint16_t *gain;             // ROWS_NORM: bf16 [k]
    void *total;                      // ROWS_NORM: x + delta (may be x)
    int8_t *q;
    float *scale;
    int64_t ldx, ld_delta, ld_total, ldq;
    int k, tile;                      // ROWS_GATE: columns of a gate tile (its up tile follows), k = one tile
    double eps;
};

__device__ __forceinline__ uint16_t to_bf16(float f) { return f != f ? (uint16_t)0x7FC0 : f32_to_bf16(f); }

// 8 values of a row from column `at`; VEC: 16-byte loads (at and the row are multiples of 8 elements), else n of them singly
template <bool BF16, bool VEC>
__device__ __forceinline__ void load8(const void *row, int64_t at, int n, float v[8]) {
    if constexpr (VEC) {
        if (n == 8) {
            if constexpr (BF16) {
                const uint4 u = *reinterpret_cast<const uint4 *>((const uint16_t *)row + at);
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    v[2 * e] = __uint_as_float(w[e] << 16);
                    v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
                }
            } else {
                const float4 a = *reinterpret_cast<const float4 *>((const float *)row + at);
                const float4 b = *reinterpret_cast<const float4 *>((const float *)row + at + 4);
                v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
            }
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        if constexpr (BF16) v[e] = e < n ? bf16_to_f32(((const uint16_t *)row)[at + e]) : 0.f;
        else v[e] = e < n ? ((const float *)row)[at + e] : 0.f;
    }
}
template <bool BF16, bool VEC>
__device__ __forceinline__ void store8(void *row, int64_t at, int n, const float v[8]) {
    if constexpr (VEC) {
        if (n == 8) {
            if constexpr (BF16) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; e++) w[e] = (uint32_t)to_bf16(v[2 * e]) | ((uint32_t)to_bf16(v[2 * e + 1]) << 16);
                *reinterpret_cast<uint4 *>((uint16_t *)row + at) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                *reinterpret_cast<float4 *>((float *)row + at) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4 *>((float *)row + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (e < n) {
            if constexpr (BF16) ((uint16_t *)row)[at + e] = to_bf16(v[e]);
            else ((float *)row)[at + e] = v[e];
        }
}

__device__ __forceinline__ float gated(float g, float u) { return g / (1.0f + expf(-g)) * u; }
__device__ __forceinline__ double gated_exactly(float g, float u) { return (double)g / (1.0 + exp(-(double)g)) * (double)u; }

template <typename T>
__device__ __forceinline__ T wave_max(T v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
    return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// NV groups of 8 values per thread are held in registers.  KEEP false (rows longer than a workgroup holds; not the norm): the
// groups go round and the row is read twice, the second time mostly from cache.
template <int KIND, bool XB, bool DB, bool VEC, int NV, bool KEEP>
__global__ __launch_bounds__(1024) void rows_q8_kernel(RowsArgs a) {
    static_assert(KEEP || KIND != ROWS_NORM, "the norm holds its row");
    __shared__ float s_max[16];
    __shared__ double s_top[16], s_sum[16];
    __shared__ unsigned long long s_exact;
    const int row = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, waves = blockDim.x >> 6, k = a.k;
    const char *x = (const char *)a.x + (int64_t)row * a.ldx * (XB ? 2 : 4);
    int8_t *q = a.q + (int64_t)row * a.ldq;
    float h[NV][8], g[KIND == ROWS_NORM ? NV : 1][8];       // the row's values (ROWS_NORM: before the gain), and the gains

    // (ROWS_GATE) the gate column of value `at`; its up column is a.tile further
    auto gate_column = [&](int at) __attribute__((always_inline)) { return a.tile == 16 ? ((at >> 4) << 5) + (at & 15) : at; };
    auto one = [&](int col) __attribute__((always_inline)) {
        return XB ? bf16_to_f32(((const uint16_t *)x)[col]) : ((const float *)x)[col];
    };
    auto exactly = [&](int at) __attribute__((always_inline)) {
        const int col = gate_column(at);
        return gated_exactly(one(col), one(col + a.tile));
    };

    auto fetch = [&](int v, int at) __attribute__((always_inline)) {
        const int n = min(max(k - at, 0), 8);
        if (KIND == ROWS_GATE && n > 0) {
            float u[8];
            const int col = gate_column(at);
            load8<XB, VEC>(x, col, n, h[v]);
            load8<XB, VEC>(x, col + a.tile, n, u);
#pragma unroll
            for (int e = 0; e < 8; e++) h[v][e] = gated(h[v][e], u[e]);
        } else if (n > 0) {
            load8<XB, VEC>(x, at, n, h[v]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) h[v][e] = 0.f;
        }
        return n;
    };

    float top32 = 0.f;
    double top = 0.0, sum = 0.0;
    bool bad = false;
    const int per_turn = NV * blockDim.x * 8, turns = KEEP ? 1 : (k + per_turn - 1) / per_turn;
    for (int turn = 0; turn < turns; turn++) {
#pragma unroll
        for (int v = 0; v < NV; v++) {
            const int at = turn * per_turn + (v * blockDim.x + tid) * 8;
            const int n = fetch(v, at);
            if constexpr (KIND == ROWS_NORM) {
                if (n > 0) {
                    load8<true, VEC>(a.gain, at, n, g[v]);
                    if (a.delta) {
                        float d[8];
                        load8<DB, VEC>((const char *)a.delta + (int64_t)row * a.ld_delta * (DB ? 2 : 4), at, n, d);
#pragma unroll
                        for (int e = 0; e < 8; e++) {
                            h[v][e] += d[e];
                            if constexpr (XB) h[v][e] = bf16_to_f32(to_bf16(h[v][e]));     // (what is stored is what is normalised)
                        }
                        store8<XB, VEC>((char *)a.total + (int64_t)row * a.ld_total * (XB ? 2 : 4), at, n, h[v]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++) g[v][e] = 0.f;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {
                if constexpr (KIND == ROWS_NORM) {
                    const double hd = h[v][e], p = fabs(hd * (double)g[v][e]);
                    bad |= !(p <= 1.7976931348623157e308);
                    top = fmax(top, p);
                    sum = fma(hd, hd, sum);
                } else {
                    const float p = fabsf(h[v][e]);
                    bad |= !(p <= 3.4028235e38f);
                    top32 = fmaxf(top32, p);
                }
            }
        }
    }
    // the row's maximum (and sum of squares); a bad row's is NaN
    if constexpr (KIND == ROWS_NORM) {
        top = wave_max(top);
        sum = wave_sum(sum);
    } else {
        top32 = wave_max(top32);
    }
    const bool wave_bad = __builtin_amdgcn_ballot_w64(bad) != 0;
    if ((tid & 63) == 0) {
        s_max[wave] = wave_bad ? __builtin_nanf("") : top32;
        s_top[wave] = top;
        s_sum[wave] = sum;
    }
    if (tid == 0) s_exact = 0;
    __syncthreads();
    top32 = 0.f;
    top = sum = 0.0;
    bad = false;
    for (int w = 0; w < waves; w++) {
        bad |= s_max[w] != s_max[w];
        top32 = fmaxf(top32, s_max[w]);
        top = fmax(top, s_top[w]);
        sum += s_sum[w];
    }
    if constexpr (KIND == ROWS_NORM) top32 = (float)top;
    else top = top32;
    const bool in_range = top32 >= PLAIN_RANGE_LO && top32 <= PLAIN_RANGE_HI;
    if constexpr (KIND == ROWS_GATE) {
        // the largest value in double: of those that fp32 has within its error of its largest
        const float near = in_range ? top32 * (1.0f - 1e-5f) : 0.f;
        double best = 0.0;
        for (int turn = 0; turn < turns; turn++)
#pragma unroll
            for (int v = 0; v < NV; v++) {
                const int at = turn * per_turn + (v * blockDim.x + tid) * 8;
                if constexpr (!KEEP) fetch(v, at);
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (at + e < k && fabsf(h[v][e]) >= near) best = fmax(best, fabs(exactly(at + e)));
            }
        if (best > 0.0) atomicMax(&s_exact, (unsigned long long)__double_as_longlong(best));
        __syncthreads();
        top = __longlong_as_double((long long)s_exact);
    }
    if (tid == 0) {
        double s = top / 127.0;
        if constexpr (KIND == ROWS_NORM) s /= sqrt(sum / (double)k + a.eps);
        a.scale[row] = bad ? __builtin_nanf("") : top == 0.0 ? 0.f : (float)s;
    }
    const bool zero = bad || top == 0.0;
    const float c32 = 127.0f / top32;
    auto code = [&](int v, int e, int at) __attribute__((always_inline)) {
        float p32 = h[v][e];
        if constexpr (KIND == ROWS_NORM) p32 *= g[v][e];
        const float t = p32 * c32;
        float r = rintf(t);
        if (!in_range || fabsf(t - r) > 0.5f - ROUND_MARGIN) {
            if constexpr (KIND == ROWS_GATE) {
                r = at + e < k ? (float)rint(exactly(at + e) * 127.0 / top) : 0.f;
            } else {
                double p = h[v][e];
                if constexpr (KIND == ROWS_NORM) p *= (double)g[v][e];
                const double m = fabs(p), low = floor(m * (127.0 / top)), off = fma(-(2.0 * low + 1.0), top, 254.0 * m);
                const double up = off > 0.0 || (off == 0.0 && ((int)low & 1)) ? low + 1.0 : low;
                r = (float)copysign(up, p);
            }
        }
        return zero ? 0 : (int)r;
    };
    for (int turn = 0; turn < turns; turn++)
#pragma unroll
        for (int v = 0; v < NV; v++) {
            const int at = turn * per_turn + (v * blockDim.x + tid) * 8;
            if constexpr (!KEEP) fetch(v, at);
            const int n = min(max(k - at, 0), 8);
            if (n <= 0) continue;
            int c[8];
#pragma unroll
            for (int e = 0; e < 8; e++) c[e] = code(v, e, at);
            if (VEC && n == 8) {
                uint2 w;
                w.x = (c[0] & 255) | (c[1] & 255) << 8 | (c[2] & 255) << 16 | (uint32_t)c[3] << 24;
                w.y = (c[4] & 255) | (c[5] & 255) << 8 | (c[6] & 255) << 16 | (uint32_t)c[7] << 24;
                *reinterpret_cast<uint2 *>(q + at) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (e < n) q[at + e] = (int8_t)c[e];
            }
        }
}

// ---------------------------------------------------------------------------------------
#define ROWS_HELD 4                    // groups of 8 values a thread holds at most
template <int KIND, bool XB, bool DB, bool VEC>
static void launch_rows_nv(const RowsArgs &a, int m, hipStream_t s) {
    const int groups = (a.k + 7) / 8, held = (groups + 1023) / 1024;
    const int nv = held <= 1 ? 1 : held <= 2 ? 2 : 4;
    const int threads = min(1024, ((groups + nv - 1) / nv + 63) / 64 * 64);
    if (nv == 1) hipLaunchKernelGGL((rows_q8_kernel<KIND, XB, DB, VEC, 1, true>), dim3(m), dim3(threads), 0, s, a);
    else if (nv == 2) hipLaunchKernelGGL((rows_q8_kernel<KIND, XB, DB, VEC, 2, true>), dim3(m), dim3(threads), 0, s, a);
    else if constexpr (KIND != ROWS_NORM) {
        if (held <= ROWS_HELD) hipLaunchKernelGGL((rows_q8_kernel<KIND, XB, DB, VEC, 4, true>), dim3(m), dim3(threads), 0, s, a);
        else hipLaunchKernelGGL((rows_q8_kernel<KIND, XB, DB, VEC, 2, false>), dim3(m), dim3(1024), 0, s, a);
    }
}
template <int KIND, bool XB, bool DB>
static void launch_rows(const RowsArgs &a, int m, bool vec, hipStream_t s) {
    if (vec) launch_rows_nv<KIND, XB, DB, true>(a, m, s);
    else launch_rows_nv<KIND, XB, DB, false>(a, m, s);
}

// (a single row has no stride)
static bool aligned(const void *p, int64_t ld, int64_t size, int m, int to) { return (uintptr_t)p % to == 0 && (m == 1 || ld * size % to == 0); }
static bool type_ok(int32_t t) { return t == BITA_F32 || t == BITA_BF16; }
static int64_t type_size(int32_t t) { return t == BITA_BF16 ? 2 : 4; }

extern "C" int bita_quantize_rows(const void *d_x, int32_t x_type, int32_t m_rows, int64_t k, int64_t ldx, int8_t *d_q, int64_t ldq,
                                  float *d_scale, void *stream) {
    if (!d_x || !d_q || !d_scale || m_rows <= 0 || k <= 0 || !type_ok(x_type) || ldx < k || ldq < k)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_quantize_rows: bad argument");
    if (k > BITA_Q8_MAX_K) return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_quantize_rows: k %lld, at most %d", (long long)k, BITA_Q8_MAX_K);
    RowsArgs a = {};
    a.x = d_x; a.q = d_q; a.scale = d_scale; a.ldx = ldx; a.ldq = ldq; a.k = (int)k;
    const bool vec = aligned(d_x, ldx, type_size(x_type), m_rows, 16) && aligned(d_q, ldq, 1, m_rows, 8);
    if (x_type == BITA_BF16) launch_rows<ROWS_PLAIN, true, false>(a, m_rows, vec, (hipStream_t)stream);
    else launch_rows<ROWS_PLAIN, false, false>(a, m_rows, vec, (hipStream_t)stream);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}

extern "C" int bita_silu_mul_q8(const void *d_gate_up, int32_t x_type, int32_t m_rows, int64_t d_ffn, int64_t ldx, int32_t tile,
                                int8_t *d_q, int64_t ldq, float *d_scale, void *stream) {
    if (!d_gate_up || !d_q || !d_scale || m_rows <= 0 || d_ffn <= 0 || !type_ok(x_type) || ldx < 2 * d_ffn || ldq < d_ffn)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_silu_mul_q8: bad argument");
    if ((tile != 0 && tile != 16) || (tile == 16 && d_ffn % 16))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_silu_mul_q8: tile must be 0 (all gate columns first) or 16 (d_ffn a multiple of 16)");
    if (d_ffn > BITA_Q8_MAX_K) return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_silu_mul_q8: d_ffn %lld, at most %d", (long long)d_ffn, BITA_Q8_MAX_K);
    RowsArgs a = {};
    a.x = d_gate_up; a.q = d_q; a.scale = d_scale; a.ldx = ldx; a.ldq = ldq; a.k = (int)d_ffn; a.tile = tile ? tile : (int)d_ffn;
    const int64_t size = type_size(x_type);
    const bool vec = aligned(d_gate_up, ldx, size, m_rows, 16) && a.tile * size % 16 == 0 && aligned(d_q, ldq, 1, m_rows, 8);
    if (x_type == BITA_BF16) launch_rows<ROWS_GATE, true, false>(a, m_rows, vec, (hipStream_t)stream);
    else launch_rows<ROWS_GATE, false, false>(a, m_rows, vec, (hipStream_t)stream);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}

extern "C" int bita_norm_q8(const void *d_x, int32_t x_type, int32_t m_rows, int64_t d, int64_t ldx, const void *d_delta,
                            int32_t delta_type, int64_t ld_delta, const void *d_gain, float eps, void *d_total, int64_t ld_total,
                            int8_t *d_q, int64_t ldq, float *d_scale, void *stream) {
    if (!d_x || !d_gain || !d_q || !d_scale || m_rows <= 0 || d <= 0 || !type_ok(x_type) || ldx < d || ldq < d || !(eps >= 0.f) ||
        (d_delta && (!type_ok(delta_type) || ld_delta < d || !d_total || ld_total < d)))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_norm_q8: bad argument");
    if (d > 1024 * RMS_MAX_CHUNKS)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_norm_q8: d %lld, at most %d", (long long)d, 1024 * RMS_MAX_CHUNKS);
    if (d_total == d_x && d_delta && m_rows > 1 && ld_total != ldx)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_norm_q8: d_total is d_x with another row stride");
    RowsArgs a = {};
    a.x = d_x; a.delta = d_delta; a.gain = (const uint16_t *)d_gain; a.total = d_total; a.q = d_q; a.scale = d_scale;
    a.ldx = ldx; a.ld_delta = ld_delta; a.ld_total = ld_total; a.ldq = ldq; a.k = (int)d; a.eps = (double)eps;
    const int64_t size = type_size(x_type);
    const bool vec = aligned(d_x, ldx, size, m_rows, 16) && (uintptr_t)d_gain % 16 == 0 && aligned(d_q, ldq, 1, m_rows, 8) &&
                     (!d_delta || (aligned(d_delta, ld_delta, type_size(delta_type), m_rows, 16) && aligned(d_total, ld_total, size, m_rows, 16)));
    hipStream_t s = (hipStream_t)stream;
    const bool db = d_delta && delta_type == BITA_BF16;
    if (x_type == BITA_BF16) {
        if (db) launch_rows<ROWS_NORM, true, true>(a, m_rows, vec, s);
        else launch_rows<ROWS_NORM, true, false>(a, m_rows, vec, s);
    } else {
        if (db) launch_rows<ROWS_NORM, false, true>(a, m_rows, vec, s);
        else launch_rows<ROWS_NORM, false, false>(a, m_rows, vec, s);
    }
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}
