// Queries and keys made ready for attention: RMSNorm of every head with a gain, and the rotation by the row's position, in one pass
// over a QKV product.  h = x / sqrt(mean(x^2) + eps) * gain over a head's values, then (h_i, h_{i+d/2}) turned by the angle of (pos, i).
//
// A thread holds 8 neighbouring values of a head's first half and the 8 they rotate with of the second (16-byte accesses in bf16), so a head is 8
// (4) threads whose sums of squares meet in three (two) steps inside a row of lanes, and nothing else crosses a lane.  What bounds it is
// what it moves, each value read and written once: 8192 rows of 64 + 8 heads of 128 in bf16, 306 MB, 59.8 us, 5.1 TB/s, a copy's rate (with 8-byte accesses and 1, 2 or
// 4 heads a thread 72.5, 70.4 and 76.3 us); at a row or two, the launch and two round trips to memory (position, then table): 2.8 us.
#include "common.h"
#include <cmath>
#include <type_traits>

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

__device__ __forceinline__ void nr_load(const float *p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void nr_load(const uint16_t *p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
// f over the 4 or 8 neighbouring lanes that hold a head: the lane 1 away, 2 away, and the mirrored one of the other four
template <int LANES, typename F>
__device__ __forceinline__ float nr_over_head(float x, F &&f) {
    auto other = [&](auto ctrl) __attribute__((always_inline)) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, false));
    };
    x = f(x, other(std::integral_constant<int, 0xB1>{}));                       // quad_perm 1 0 3 2
    x = f(x, other(std::integral_constant<int, 0x4E>{}));                       // quad_perm 2 3 0 1
    if constexpr (LANES == 8) x = f(x, other(std::integral_constant<int, 0x141>{}));    // row_half_mirror
    return x;
}
// a head's values over its threads: times gain / sqrt(mean of squares + eps)
template <int HD>
__device__ __forceinline__ void nr_norm(float (&lo)[8], float (&hi)[8], const uint16_t *gain, float eps) {
    constexpr int LANES = HD / 16;
    const auto add = [](float x, float y) { return x + y; };
    float ss = 0.f, gl[8], gh[8];
    nr_load(gain, gl);
    nr_load(gain + HD / 2, gh);
#pragma unroll
    for (int e = 0; e < 8; e++) ss += lo[e] * lo[e] + hi[e] * hi[e];
    ss = nr_over_head<LANES>(ss, add);
    float r = 1.0f / sqrtf(ss * (1.0f / HD) + eps);
    if (!(ss <= 1e37f) || (ss < 1e-30f && eps < 1e-20f)) {
        // Squares beyond fp32's range (too small ones matter where eps is no larger), infinities, NaN: the same with the head, and sqrt(eps), divided by a
        // power of two near its largest value.  (A head's threads agree.)
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) top = fmaxf(top, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
        top = nr_over_head<LANES>(top, [](float x, float y) { return fmaxf(x, y); });
        const int k = __builtin_amdgcn_frexp_expf(top);
        ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            lo[e] = ldexpf(lo[e], -k);
            hi[e] = ldexpf(hi[e], -k);
            ss += lo[e] * lo[e] + hi[e] * hi[e];
        }
        ss = nr_over_head<LANES>(ss, add);
        const float t = ldexpf(sqrtf(eps), -k);
        r = t > 1e15f ? 1.0f / t : 1.0f / sqrtf(ss * (1.0f / HD) + t * t);
    }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        lo[e] = lo[e] * r * gl[e];
        hi[e] = hi[e] * r * gh[e];
    }
}
// (the conversion instruction rounds to nearest even and keeps NaNs)
__device__ __forceinline__ uint4 nr_bf16x8(const float (&v)[8]) {
    typedef __attribute__((ext_vector_type(8))) float f8;
    const f8 f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
    return __builtin_bit_cast(uint4, __builtin_convertvector(f, bf16x8));
}

template <typename T, int HD>
__global__ __launch_bounds__(NR_THREADS) void qk_norm_rope_kernel(NormRopeArgs a) {
    constexpr int LANES = HD / 16, SLOTS = NR_THREADS / LANES;
    const int j = threadIdx.x % LANES * 8, head = blockIdx.y * SLOTS + threadIdx.x / LANES;
    const int n_rot = a.Hq + a.Hkv;
    if (head >= n_rot + (a.v ? a.Hkv : 0)) return;
    const bool is_q = head < a.Hq, is_v = head >= n_rot;
    const uint16_t *gain = is_v ? nullptr : is_q ? a.q_gain : a.k_gain;
    uint16_t *out = j + (is_q ? a.q + head * a.q_head : is_v ? a.v + (head - n_rot) * a.v_head : a.k + (head - a.Hq) * a.k_head);
    const int64_t ld = is_q ? a.ldq : is_v ? a.ldv : a.ldk;
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
        const T *src = reinterpret_cast<const T *>(a.x) + row * a.ldx + (int64_t)head * HD + j;
        const int p = min(max(a.pos[row], 0), a.max_pos - 1);
        float lo[8], hi[8];
        nr_load(src, lo);
        nr_load(src + HD / 2, hi);
        if (!is_v) {
            float c[8], s[8];
            nr_load(a.cos + (int64_t)p * (HD / 2) + j, c);
            nr_load(a.sin + (int64_t)p * (HD / 2) + j, s);
            if (gain) nr_norm<HD>(lo, hi, gain + j, a.eps);
#pragma unroll
            for (int e = 0; e < 8; e++) rope_pair(lo[e], hi[e], c[e], s[e]);
        }
        uint16_t *dst = out + row * ld;
        *reinterpret_cast<uint4 *>(dst) = nr_bf16x8(lo);
        *reinterpret_cast<uint4 *>(dst + HD / 2) = nr_bf16x8(hi);
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
    if ((m_rows && (!d_x || !d_pos || !d_q || !d_k)) || !d_cos || !d_sin || m_rows < 0 || n_heads <= 0 || n_kv_heads <= 0 || max_pos <= 0 || !(eps >= 0.f) || !std::isfinite(eps))
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
    const int per_wg = NR_THREADS * 16 / head_dim, used = n_heads + (d_v ? 2 : 1) * n_kv_heads;
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
