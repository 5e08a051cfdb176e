// The product of 8-bit integers with scales: Y[m][n] = (sum_k A[m][k] W[n][k]) sa[m] sw[n], sums in 32-bit integers.
#include "common.h"

typedef __attribute__((ext_vector_type(4))) int i32x4;

// 1 KiB block of rows 16t.. and k 64s.. of a packed weight: lane l holds W[16t + l%16][64s + 16(l/16) ..]
__global__ __launch_bounds__(256) void pack_q8_kernel(const int8_t *__restrict__ src, int64_t n_rows, int64_t k, int64_t ld,
                                                      uint4 *__restrict__ dst, int64_t tile0, int64_t tile_stride, int64_t total_tiles) {
    const int64_t t = blockIdx.x;                            // source tile
    const int lane = threadIdx.x & 63;
    const int64_t row = t * 16 + (lane & 15), steps = (k + 127) / 128 * 2;
    for (int64_t s = blockIdx.y * 4 + (threadIdx.x >> 6); s < steps; s += gridDim.y * 4) {
        const int64_t col = s * 64 + (lane >> 4) * 16;
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        if (row < n_rows && col < k) {
            const int8_t *p = src + row * ld + col;
            if (col + 16 <= k && ((uintptr_t)p & 15) == 0) {
                const uint4 v = *reinterpret_cast<const uint4 *>(p);
                w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            } else {
#pragma unroll
                for (int e = 0; e < 16; e++)
                    if (col + e < k) w[e >> 2] |= (uint32_t)(uint8_t)p[e] << (8 * (e & 3));
            }
        }
        dst[(((s >> 1) * total_tiles + tile0 + t * tile_stride) * 2 + (s & 1)) * 64 + lane] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__device__ __forceinline__ void store_out(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_out(uint16_t *p, float v) { *p = v != v ? (uint16_t)0x7FC0 : f32_to_bf16(v); }

// One 16 x 16 tile per wave, operands straight from memory.
template <typename OUT>
__global__ __launch_bounds__(256) void gemm_q8_kernel(const int8_t *__restrict__ a, int64_t lda, const float *__restrict__ sa, int m,
                                                      const i32x4 *__restrict__ w, const float *__restrict__ sw, int64_t n, int k_pairs, int k_last,
                                                      OUT *__restrict__ out, int64_t ldo) {
    const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4;
    const int64_t n_tiles = (n + 15) >> 4, tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int m0 = blockIdx.y * 16;
    if (tile >= n_tiles) return;
    const int8_t *ar = a + (int64_t)min(m0 + r, m - 1) * lda;
    i32x4 acc = {0, 0, 0, 0};
    for (int p = 0; p < k_pairs; p++)
#pragma unroll
        for (int s = 0; s < 2; s++) {
            // (columns past the row's end: anything, their weights are zero)
            const i32x4 x = *reinterpret_cast<const i32x4 *>(ar + min(p * 128 + s * 64 + c * 16, k_last));
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, w[(((int64_t)p * n_tiles + tile) * 2 + s) * 64 + lane], acc, 0, 0, 0);
        }
    const int64_t col = tile * 16 + r;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const int row = m0 + 4 * c + e;
        if (row < m && col < n) store_out(out + (int64_t)row * ldo + col, (float)acc[e] * sa[row] * sw[col]);
    }
}

extern "C" size_t bita_packed_q8_bytes(int64_t n_rows, int64_t k) {
    if (n_rows <= 0 || k <= 0) return 0;
    return (size_t)((n_rows + 15) / 16) * (size_t)((k + 127) / 128) * 2048;
}

extern "C" int bita_pack_weight_q8(const int8_t *d_src, int64_t n_rows, int64_t k, int64_t ld, void *d_dst, int64_t dst_total_rows,
                                   int64_t dst_tile0, int64_t dst_tile_stride, void *stream) {
    if (!d_src || !d_dst || n_rows <= 0 || k <= 0 || ld < k || dst_tile0 < 0 || dst_tile_stride < 1 || (uintptr_t)d_dst % 16)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_pack_weight_q8: bad argument");
    const int64_t tiles = (n_rows + 15) / 16, total = (dst_total_rows + 15) / 16, last = dst_tile0 + (tiles - 1) * dst_tile_stride;
    if (last >= total)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_pack_weight_q8: source tiles do not fit %lld destination rows", (long long)dst_total_rows);
    if (n_rows % 16 && last != total - 1)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_pack_weight_q8: %lld rows end inside a tile that is not the destination's last", (long long)n_rows);
    if (k > BITA_Q8_MAX_K || tiles > INT32_MAX)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_pack_weight_q8: %lld rows of %lld", (long long)n_rows, (long long)k);
    hipLaunchKernelGGL(pack_q8_kernel, dim3((unsigned)tiles, (unsigned)min((int64_t)8, (k + 255) / 256)), dim3(256), 0, (hipStream_t)stream, d_src, n_rows,
                       k, ld, (uint4 *)d_dst, dst_tile0, dst_tile_stride, total);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}

extern "C" int bita_gemm_q8(const int8_t *d_a, int64_t lda, const float *d_a_scale, int32_t m_rows, int64_t k, const void *d_w_packed,
                            const float *d_w_scale, int64_t n_rows, void *d_out, int32_t out_type, int64_t ldo, void *stream) {
    if (!d_a || !d_a_scale || !d_w_packed || !d_w_scale || !d_out || m_rows <= 0 || k <= 0 || n_rows <= 0 || ldo < n_rows ||
        (out_type != BITA_F32 && out_type != BITA_BF16))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_gemm_q8: bad argument");
    if ((uintptr_t)d_a % 16 || (uintptr_t)d_w_packed % 16 || lda % 16 || (m_rows > 1 && lda < k))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_gemm_q8: d_a, d_w_packed and lda have to be multiples of 16, lda at least k");
    if (k > BITA_Q8_MAX_K) return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_gemm_q8: k %lld, at most %d", (long long)k, BITA_Q8_MAX_K);
    const int k_pairs = (int)((k + 127) / 128), k_last = (int)((k + 15) / 16 * 16 - 16);
    const dim3 grid((unsigned)(((n_rows + 15) / 16 + 3) / 4), (unsigned)((m_rows + 15) / 16));
    hipStream_t s = (hipStream_t)stream;
    if (out_type == BITA_BF16)
        hipLaunchKernelGGL(gemm_q8_kernel<uint16_t>, grid, dim3(256), 0, s, d_a, lda, d_a_scale, m_rows, (const i32x4 *)d_w_packed, d_w_scale, n_rows, k_pairs, k_last,
                           (uint16_t *)d_out, ldo);
    else
        hipLaunchKernelGGL(gemm_q8_kernel<float>, grid, dim3(256), 0, s, d_a, lda, d_a_scale, m_rows, (const i32x4 *)d_w_packed, d_w_scale, n_rows, k_pairs, k_last,
                           (float *)d_out, ldo);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}
