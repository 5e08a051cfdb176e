// Causal attention over packed prompts: o_i = sum_{j <= i} softmax_j(q_i k_j / sqrt(d)) v_j inside every sequence.
//
// A workgroup owns 128 queries of one head, 32 a wave, and walks the keys in tiles of 64 up to its last query, with a running maximum
// and sum per query.
//  * S^T = K Q^T by 32 x 32 x 16 matrix instructions: a lane has 32 of its query's 64 scores, the other half wave the rest, so a maximum or a sum
//    crosses lanes once.  The layout of S^T is the B operand of O^T = V^T P^T when that takes the keys in the order in which S^T
//    holds them (lane half h: keys 8 i + 4 h + 0..3): the probabilities stay in registers.
//  * K and V tiles go from memory to LDS without passing registers, into one of two buffers, while the other is multiplied; one
//    barrier a tile.  Rows are swizzled by 16-byte columns on the way (by where a lane fetches from: LDS takes them in lane order),
//    K is read back by rows, V by transposed reads.
//  * Key tiles before a wave's queries need no mask.  Workgroups start with the longest walks.
#include "nonfinite.h"
#include <cmath>

#define PA_WAVES 4
#define PA_KEYS 64
#define PA_ROWS (32 * PA_WAVES)

typedef __attribute__((ext_vector_type(16))) float f32x16;

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t ldq, q_head, ldk, k_head, ldv, v_head, ldo;
    const int32_t *cu;
    int n_seqs, n_tokens, Hq, qpk;
    float scale_log2;
    uint16_t *out;
};

__device__ __forceinline__ float pa_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ uint32_t pa_pk_bf16(float a, float b) {
    typedef __attribute__((ext_vector_type(2))) float f2;
    typedef __attribute__((ext_vector_type(2))) __bf16 b2;
    const f2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
}
// the other half wave's value
__device__ __forceinline__ float pa_other_half(float x) {
    typedef __attribute__((ext_vector_type(2))) unsigned u2;
    const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// The tile's sequence, its first token and length, and the tile's number inside it, from the sequences' ends: tiles are counted over
// the sequences, 64 of them a step.  false: no such tile.
__device__ __forceinline__ bool pa_find(const PromptArgs &a, int tile, int &start, int &len, int &mine) {
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        const int b = b0 + lane;
        int s = 0, n = 0;
        if (b < a.n_seqs) {
            s = min(max(a.cu[b], 0), a.n_tokens);
            n = min(max(a.cu[b + 1], s), a.n_tokens) - s;
        }
        const int tiles = (n + PA_ROWS - 1) / PA_ROWS;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int other = __shfl_up(upto, d);
            if (lane >= d) upto += other;
        }
        const int all = __shfl(upto, 63);
        if (tile < all) {
            const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > tile));
            start = __builtin_amdgcn_readlane(s, at);
            len = __builtin_amdgcn_readlane(n, at);
            mine = tile - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(tiles, at));
            return true;
        }
        tile -= all;
    }
    return false;
}

template <int HD>
__global__ __launch_bounds__(PA_WAVES * 64, 2) void prompt_attn_kernel(PromptArgs a) {
    constexpr int KS = HD / 16, NT = HD / 32, GPR = HD / 8, RPI = 64 / GPR;             // k-steps, head tiles, granules a row, rows a load instruction
    constexpr int TILE = PA_KEYS * HD * 2, LOADS = PA_KEYS / RPI / PA_WAVES;            // bytes of a K (or V) tile; load instructions a wave
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];                // [2][K | V]
    const int lane = threadIdx.x & 63, hf = lane >> 5, c = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j = blockIdx.x % a.Hq;
    const int head = a.Hq % 8 == 0 ? (j & 7) * (a.Hq >> 3) + (j >> 3) : j;              // an XCD (ids go round) takes neighbouring heads
    int start, len, tile;
    if (!pa_find(a, blockIdx.x / a.Hq, start, len, tile)) return;
    tile = (len + PA_ROWS - 1) / PA_ROWS - 1 - tile;                                    // the longest walk first
    const int q0 = tile * PA_ROWS + wave * 32, qi = q0 + c, kvh = head / a.qpk;         // of the wave, of the lane: inside the sequence
    const int64_t qrow = start + min(qi, len - 1);

    bf16x8 qf[KS];
#pragma unroll
    for (int s = 0; s < KS; s++)
        qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(a.q + qrow * a.ldq + head * a.q_head + 16 * s + 8 * hf));

    const int keys = min(len, (tile + 1) * PA_ROWS), n_tiles = (keys + PA_KEYS - 1) / PA_KEYS;
    auto k_swizzle = [](int r) __attribute__((always_inline)) { return HD == 128 ? r & 15 : (r >> 1) & 7; };
    auto v_swizzle = [](int r) __attribute__((always_inline)) { return HD == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); };
    const uint16_t *kbase = a.k + (int64_t)start * a.ldk + kvh * a.k_head, *vbase = a.v + (int64_t)start * a.ldv + kvh * a.v_head;
    auto fetch = [&](int t, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int piece = wave * LOADS + i, r = piece * RPI + lane / GPR, p = lane % GPR;
            const int64_t key = min(t * PA_KEYS + r, len - 1);
            const uint16_t *ks = kbase + key * a.ldk + (p ^ k_swizzle(r)) * 8, *vs = vbase + key * a.ldv + (p ^ v_swizzle(r)) * 8;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)ks,
                                             (__attribute__((address_space(3))) void *)(smem + buf * 2 * TILE + piece * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)vs,
                                             (__attribute__((address_space(3))) void *)(smem + buf * 2 * TILE + TILE + piece * 1024), 16, 0, 0);
        }
    };

    f32x16 o[NT];
#pragma unroll
    for (int n = 0; n < NT; n++) o[n] = f32x16{};
    float m_run = -INFINITY, l_run = 0.f;

    fetch(0, 0);
    for (int t = 0; t < n_tiles; t++) {
        __builtin_amdgcn_s_waitcnt(0x0F70);                                             // vmcnt(0): this wave's part of the tile is in LDS
        __syncthreads();                                                                // everyone's is, and everyone has read the other buffer
        if (t + 1 < n_tiles) fetch(t + 1, (t + 1) & 1);
        const int key0 = t * PA_KEYS;
        if (key0 > q0 + 31 || q0 >= len) continue;                                      // nothing here for this wave's queries
        const unsigned char *kt = smem + (t & 1) * 2 * TILE, *vt = kt + TILE;
        f32x16 s[2];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            s[h] = f32x16{};
#pragma unroll
            for (int ks = 0; ks < KS; ks++) {
                const int r = 32 * h + c;
                const bf16x8 kf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(kt + r * (HD * 2) + (((2 * ks + hf) ^ k_swizzle(r)) * 16)));
                s[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], s[h], 0, 0, 0);
            }
        }
        const bool need_mask = key0 + PA_KEYS - 1 > q0;
        if (need_mask) {
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int e = 0; e < 16; e++) s[h][e] = key0 + 32 * h + 8 * (e >> 2) + 4 * hf + (e & 3) <= qi ? s[h][e] : -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; e++) mx = fmaxf(mx, fmaxf(s[0][e], s[1][e]));
        if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
            const float m_new = fmaxf(m_run, fmaxf(mx, pa_other_half(mx)));
            const float alpha = m_new == -INFINITY ? 1.f : pa_exp2((m_run - m_new) * a.scale_log2);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int n = 0; n < NT; n++) o[n] *= alpha;
        }
        const float base = m_run == -INFINITY ? 0.f : m_run * a.scale_log2;
        float ps = 0.f;
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int e = 0; e < 16; e++) {
                s[h][e] = pa_exp2(__builtin_fmaf(s[h][e], a.scale_log2, -base));
                ps += s[h][e];
            }
        l_run += ps;
#pragma unroll
        for (int kk = 0; kk < PA_KEYS / 16; kk++) {
            const int h = kk >> 1, e0 = 8 * (kk & 1);
            uint32_t pk[4];
#pragma unroll
            for (int e = 0; e < 4; e++) pk[e] = pa_pk_bf16(s[h][e0 + 2 * e], s[h][e0 + 2 * e + 1]);
            const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3]));
#pragma unroll
            for (int n = 0; n < NT; n++) {
                typedef __attribute__((ext_vector_type(4))) short s4;
                typedef __attribute__((ext_vector_type(8))) short s8;
                typedef __attribute__((address_space(3))) s4 *lds_s4;
                s4 half[2];
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    // four keys of 16 columns a group of 16 lanes: this lane names one key's four columns and gets its own column of the four keys
                    const int r = 16 * kk + 8 * x + 4 * hf + ((c & 15) >> 2), col = 32 * n + (c & 16) + 4 * (c & 3);
                    half[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(vt + r * (HD * 2) + (((col >> 3) ^ v_swizzle(r)) * 16) + (col & 4) * 2));
                }
                bf16x8 vf = __builtin_bit_cast(bf16x8, s8{half[0][0], half[0][1], half[0][2], half[0][3], half[1][0], half[1][1], half[1][2], half[1][3]});
                if (need_mask && __builtin_amdgcn_ballot_w64(has_nonfinite(vf)) != 0) {
                    bf16x8 up, down;
                    split_nonfinite(vf, up, down);
                    uint32_t one[4];
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int key = key0 + 16 * kk + 8 * (e >> 1) + 4 * hf + 2 * (e & 1);
                        one[e] = (key <= qi ? 0x3F80u : 0u) | (key + 1 <= qi ? 0x3F800000u : 0u);
                    }
                    const bf16x8 seen = __builtin_bit_cast(bf16x8, make_uint4(one[0], one[1], one[2], one[3]));
                    const f32x16 a_up = __builtin_amdgcn_mfma_f32_32x32x16_bf16(up, seen, f32x16{}, 0, 0, 0);
                    const f32x16 a_down = __builtin_amdgcn_mfma_f32_32x32x16_bf16(down, seen, f32x16{}, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 16; e++) o[n][e] += nonfinite_term(a_up[e], a_down[e]);
                }
                o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[n], 0, 0, 0);
            }
        }
    }
    if (qi >= len) return;
    const float l = l_run + pa_other_half(l_run), inv = 1.0f / l;
    uint16_t *dst = a.out + qrow * a.ldo + (int64_t)head * HD + 4 * hf;
#pragma unroll
    for (int n = 0; n < NT; n++)
#pragma unroll
        for (int i = 0; i < 4; i++)
            *reinterpret_cast<uint2 *>(dst + 32 * n + 8 * i) = make_uint2(pa_pk_bf16(o[n][4 * i] * inv, o[n][4 * i + 1] * inv),
                                                                          pa_pk_bf16(o[n][4 * i + 2] * inv, o[n][4 * i + 3] * inv));
}

extern "C" int bita_prompt_attention(const void *d_q, int64_t ldq, int64_t q_head_stride, const void *d_k, int64_t ldk, int64_t k_head_stride,
                                     const void *d_v, int64_t ldv, int64_t v_head_stride, const int32_t *d_cu_seqlens, int32_t n_seqs, int32_t n_tokens,
                                     int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, void *d_out, int64_t ldo, void *stream) {
    const char *who = "bita_prompt_attention";
    if (!d_q || !d_k || !d_v || !d_cu_seqlens || !d_out || n_seqs <= 0 || n_tokens < 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads)
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: null argument, non-positive or inconsistent size", who);
    if (head_dim != 64 && head_dim != 128) return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128", who);
    if (ldq < 0 || ldk < 0 || ldv < 0 || q_head_stride < 0 || k_head_stride < 0 || v_head_stride < 0 || ldo < (int64_t)n_heads * head_dim)
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: negative stride, or output rows of %lld values %lld apart", who, (long long)n_heads * head_dim, (long long)ldo);
    if ((ldq | ldk | ldv | q_head_stride | k_head_stride | v_head_stride | ldo) & 7 ||
        ((uintptr_t)d_q | (uintptr_t)d_k | (uintptr_t)d_v | (uintptr_t)d_out) & 15)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: strides must be multiples of 8 elements, pointers of 16 bytes", who);
    const int64_t tiles = (int64_t)n_tokens / PA_ROWS + n_seqs, wgs = tiles * n_heads;          // no tiling of the sequences has more
    if (wgs > (int64_t)((1ull << 32) / (PA_WAVES * 64)) - 1)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: %lld workgroups", who, (long long)wgs);
    if (n_tokens == 0) return BITA_OK;
    const PromptArgs a = {(const uint16_t *)d_q, (const uint16_t *)d_k, (const uint16_t *)d_v, ldq, q_head_stride, ldk, k_head_stride, ldv, v_head_stride, ldo,
                          d_cu_seqlens, n_seqs, n_tokens, n_heads, n_heads / n_kv_heads, 1.4426950408889634f / sqrtf((float)head_dim), (uint16_t *)d_out};
    hipStream_t s = (hipStream_t)stream;
    if (head_dim == 128) hipLaunchKernelGGL((prompt_attn_kernel<128>), dim3((unsigned)wgs), dim3(PA_WAVES * 64), 4 * PA_KEYS * 128 * 2, s, a);
    else hipLaunchKernelGGL((prompt_attn_kernel<64>), dim3((unsigned)wgs), dim3(PA_WAVES * 64), 4 * PA_KEYS * 64 * 2, s, a);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}
