// Queries and keys made ready for attention: RMSNorm of every head with a gain, and the rotation by the row's position, in one pass
// over a QKV product.  h = x / sqrt(mean(x^2) + eps) * gain over a head's values, then (h_i, h_{i+d/2}) turned by the angle of (pos, i).
//
// A thread holds 4 neighbouring values of a head's first half and the 4 they rotate with of the second, so a head is 16 (8)
// threads whose sums of squares meet in four (three) lane exchanges, and nothing else crosses a lane.  What bounds it is what it
// moves, each value read and written once; at a row or two, the launch and two round trips to memory (position, then table).
#include "common.h"
#include <cmath>

#define NR_THREADS 256
#define NR_GRID_ROWS (1 << 20)          // rows a launch has workgroups of their own for; more are walked

struct NormRopeArgs {
    const void *x;
    int64_t ldx;
    int M, Hq, Hkv, max_pos;
    const uint16_t *q_gain, *k_gain;
    float eps;
    const int32_t *pos;
    const float *cos, *sin;
    uint16_t *q, *k, *v;
    int64_t ldq, q_head, ldk, k_head, ldv, v_head;
};

__device__ __forceinline__ void nr_load(const float *p, float (&v)[4]) {
    const float4 a = *reinterpret_cast<const float4 *>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ void nr_load(const uint16_t *p, float (&v)[4]) {
    const uint2 a = *reinterpret_cast<const uint2 *>(p);
    v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xFFFF0000u);
    v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xFFFF0000u);
}
// (the conversion instruction rounds to nearest even and keeps NaNs)
__device__ __forceinline__ uint2 nr_bf16x4(const float (&v)[4]) {
    typedef __attribute__((ext_vector_type(4))) float f4;
    typedef __attribute__((ext_vector_type(4))) __bf16 b4;
    const f4 f = {v[0], v[1], v[2], v[3]};
    return __builtin_bit_cast(uint2, __builtin_convertvector(f, b4));
}

template <typename T, int HD>
__global__ __launch_bounds__(NR_THREADS) void qk_norm_rope_kernel(NormRopeArgs a) {
    constexpr int LANES = HD / 8, HEADS = NR_THREADS / LANES;
    const int j = threadIdx.x % LANES * 4, head = blockIdx.y * HEADS + threadIdx.x / LANES;
    const int n_heads = a.Hq + (a.v ? 2 : 1) * a.Hkv;
    if (head >= n_heads) return;
    const bool is_q = head < a.Hq, is_v = head >= a.Hq + a.Hkv;
    const uint16_t *gain = is_v ? nullptr : is_q ? a.q_gain : a.k_gain;
    uint16_t *out = is_q ? a.q : is_v ? a.v : a.k;
    const int64_t ld = is_q ? a.ldq : is_v ? a.ldv : a.ldk;
    out += is_q ? head * a.q_head : is_v ? (head - a.Hq - a.Hkv) * a.v_head : (head - a.Hq) * a.k_head;
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
        const T *src = reinterpret_cast<const T *>(a.x) + row * a.ldx + (int64_t)head * HD + j;
        float lo[4], hi[4];
        nr_load(src, lo);
        nr_load(src + HD / 2, hi);
        if (!is_v) {
            const int p = min(max(a.pos[row], 0), a.max_pos - 1);
            float c[4], s[4];
            nr_load(a.cos + (int64_t)p * (HD / 2) + j, c);
            nr_load(a.sin + (int64_t)p * (HD / 2) + j, s);
            if (gain) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 4; e++) ss += lo[e] * lo[e] + hi[e] * hi[e];
#pragma unroll
                for (int d = 1; d < LANES; d *= 2) ss += __shfl_xor(ss, d);
                float gl[4], gh[4];
                nr_load(gain + j, gl);
                nr_load(gain + j + HD / 2, gh);
                if (ss >= 1e-30f && ss <= 1e37f) {
                    const float r = 1.0f / sqrtf(ss * (1.0f / HD) + a.eps);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        lo[e] = lo[e] * r * gl[e];
                        hi[e] = hi[e] * r * gh[e];
                    }
                } else {                                        // squares that leave fp32's range, zeros, infinities, NaN (a head's threads agree)
                    double dd = 0.0;
#pragma unroll
                    for (int e = 0; e < 4; e++) dd += (double)lo[e] * lo[e] + (double)hi[e] * hi[e];
#pragma unroll
                    for (int d = 1; d < LANES; d *= 2) dd += __shfl_xor(dd, d);
                    const double r = 1.0 / sqrt(dd / HD + (double)a.eps);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        lo[e] = (float)(lo[e] * r * gl[e]);
                        hi[e] = (float)(hi[e] * r * gh[e]);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; e++) rope_pair(lo[e], hi[e], c[e], s[e]);
        }
        uint16_t *dst = out + row * ld + j;
        *reinterpret_cast<uint2 *>(dst) = nr_bf16x4(lo);
        *reinterpret_cast<uint2 *>(dst + HD / 2) = nr_bf16x4(hi);
    }
}

extern "C" int bita_qk_norm_rope(const void *d_x, int32_t x_type, int32_t m_rows, int64_t ldx, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                 const void *d_q_gain, const void *d_k_gain, float eps, const int32_t *d_pos, const float *d_cos, const float *d_sin,
                                 int32_t max_pos, void *d_q, int64_t ldq, int64_t q_head_stride, void *d_k, int64_t ldk, int64_t k_head_stride,
                                 void *d_v, int64_t ldv, int64_t v_head_stride, void *stream) {
    const char *who = "bita_qk_norm_rope";
    if (m_rows <= 1) ldx = ((int64_t)n_heads + 2 * (int64_t)n_kv_heads) * head_dim, ldq = ldk = ldv = 0;       // (strides of axes with one place are nobody's)
    if (n_heads == 1) q_head_stride = 0;
    if (n_kv_heads == 1) k_head_stride = v_head_stride = 0;
    if (!d_x || !d_pos || !d_cos || !d_sin || !d_q || !d_k || m_rows < 0 || n_heads <= 0 || n_kv_heads <= 0 || max_pos <= 0 || !(eps >= 0.f) || !std::isfinite(eps))
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: null argument, non-positive size or bad eps", who);
    if (x_type != BITA_F32 && x_type != BITA_BF16) return bita_set_error(BITA_ERR_INVALID_ARG, "%s: type %d", who, x_type);
    const int64_t heads = (int64_t)n_heads + 2 * (int64_t)n_kv_heads;
    if ((head_dim != 64 && head_dim != 128) || heads > 65535 * 16)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128, heads at most %d", who, 65535 * 16);
    if (ldx < heads * head_dim || ldq < 0 || ldk < 0 || ldv < 0 || q_head_stride < 0 || k_head_stride < 0 || v_head_stride < 0)
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: rows of %lld values do not fit a stride of %lld, or a negative stride", who, (long long)heads * head_dim, (long long)ldx);
    if ((ldx | ldq | ldk | q_head_stride | k_head_stride | (d_v ? ldv | v_head_stride : 0)) & 7 ||
        ((uintptr_t)d_x | (uintptr_t)d_q | (uintptr_t)d_k | (uintptr_t)d_v | (uintptr_t)d_cos | (uintptr_t)d_sin | (uintptr_t)d_q_gain | (uintptr_t)d_k_gain) & 15)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: strides must be multiples of 8 elements, pointers of 16 bytes", who);
    if (rows_overlap(head_dim, {m_rows, ldq}, {n_heads, q_head_stride}) || rows_overlap(head_dim, {m_rows, ldk}, {n_kv_heads, k_head_stride}) ||
        (d_v && rows_overlap(head_dim, {m_rows, ldv}, {n_kv_heads, v_head_stride})))
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: rows of an output overlap", who);
    if (m_rows == 0) return BITA_OK;
    const NormRopeArgs a = {d_x, ldx, m_rows, n_heads, n_kv_heads, max_pos, (const uint16_t *)d_q_gain, (const uint16_t *)d_k_gain, eps, d_pos, d_cos, d_sin,
                            (uint16_t *)d_q, (uint16_t *)d_k, (uint16_t *)d_v, ldq, q_head_stride, ldk, k_head_stride, ldv, v_head_stride};
    const int per_wg = NR_THREADS * 8 / head_dim, used = n_heads + (d_v ? 2 : 1) * n_kv_heads;
    const dim3 grid(m_rows < NR_GRID_ROWS ? m_rows : NR_GRID_ROWS, (used + per_wg - 1) / per_wg);
    hipStream_t s = (hipStream_t)stream;
    if (x_type == BITA_F32) {
        if (head_dim == 128) hipLaunchKernelGGL((qk_norm_rope_kernel<float, 128>), grid, dim3(NR_THREADS), 0, s, a);
        else hipLaunchKernelGGL((qk_norm_rope_kernel<float, 64>), grid, dim3(NR_THREADS), 0, s, a);
    } else {
        if (head_dim == 128) hipLaunchKernelGGL((qk_norm_rope_kernel<uint16_t, 128>), grid, dim3(NR_THREADS), 0, s, a);
        else hipLaunchKernelGGL((qk_norm_rope_kernel<uint16_t, 64>), grid, dim3(NR_THREADS), 0, s, a);
    }
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}
