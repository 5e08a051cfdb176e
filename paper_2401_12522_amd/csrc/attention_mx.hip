// Attention of a pass' rows over a K/V cache in 4 or 8 bits: o = softmax(q k^T / sqrt(d)) v over [prefix | cache | pass rows], the
// prefix seen by mask rows, the pass rows by their descendants-or-self.
//
// A K/V head's queries are one axis: R rows times the heads of its group, 16 of them a tile, whatever the number of heads.  A workgroup
// owns U tiles and a share of the keys, which its waves walk in chunks of 32, each with its own running maximum and sum; the waves' results meet
// in LDS once at the end, the shares' (where the keys are split over workgroups) in a second kernel.
//  * Codes go from memory to registers, a chunk ahead of the arithmetic, and from there to bf16 (exact: a code times a power of two) by
//    conversion instructions that apply the scale: a lane holds a quarter of a key's head, one block of 32 values (half of one at 64).
//  * The contraction over the head runs in the order in which a lane holds it: k-step s takes values 8s .. 8s+7 of every lane's
//    quarter, of the queries too, so K needs no other layout than the cache's.
//  * S^T = K Q^T leaves lane (g, c) the scores of keys 4g .. 4g+3 of either half of the chunk for query c, which is the
//    B operand of O^T = V^T P^T if that product takes the keys in the same order: probabilities stay in registers.
//  * V^T needs eight keys of one column in a lane: V goes to LDS as bf16 rows and comes back by transposed reads.  The region is the wave's own,
//    and its LDS instructions run in order, so there is no barrier in the loop.
#include "mx.h"
#include "nonfinite.h"
#include <cmath>

#define AMX_CHUNK 32
#define AMX_WAVES 4

__device__ __forceinline__ float amx_exp2(float x) { return __builtin_amdgcn_exp2f(x); }        // arguments <= 0: results below 2^-126 are zero
__device__ __forceinline__ uint32_t amx_pk_bf16(float a, float b) {
    const mx_f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, mx_bf16x2));
}
// over the lanes l, l^16, l^32, l^48
template <typename F>
__device__ __forceinline__ float amx_over_groups(float x, F &&f) {
    typedef __attribute__((ext_vector_type(2))) unsigned u2;
    u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

struct AmxArgs {
    KvMx kv;
    TemplateDev t;
    const uint16_t *q, *k_rows, *v_rows, *prompt_k, *prompt_v;
    MxRows k_at, v_at;
    const int32_t *ctx_len, *token;
    int P, R, qpk, ctx_hint, n_tiles, n_splits;                 // tiles of 16 U queries
    float scale_log2;
    float *part_o, *part_ml;
    uint16_t *out;
};

template <int HD, int U>
struct AmxCfg {
    static constexpr int KS = HD / 32, NT = HD / 16, VPL = HD / 4;      // k-steps, 16-wide tiles of the head, values a lane holds of a key
    static constexpr int V_BYTES = AMX_CHUNK * HD * 2;                  // a wave's V chunk as bf16
    static constexpr int MERGE = U * AMX_WAVES * NT * 64 * 16;
    static constexpr int ML = AMX_WAVES * V_BYTES > MERGE ? AMX_WAVES * V_BYTES : MERGE;
    static constexpr int SMEM = ML + 2 * U * AMX_WAVES * 16 * 4;
};

// one chunk's codes and scale bytes in registers: of keys c and 16 + c
template <int HD, int BITS>
struct AmxRaw {
    static constexpr int DW = HD / 4 * BITS / 32;                       // dwords of a lane's part of a key: 4 or 8 (128), 2 or 4 (64)
    uint32_t k[2][DW], v[2][DW];
    uint32_t ks[2], vs[2];
};

template <int HD, int BITS, int U>
__global__ __launch_bounds__(AMX_WAVES * 64, 2) void attn_mx_kernel(AmxArgs a) {
    using C = AmxCfg<HD, U>;
    using Raw = AmxRaw<HD, BITS>;
    constexpr int KS = C::KS, NT = C::NT, VPL = C::VPL, DW = Raw::DW, W = AMX_WAVES;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // The tiles that read the same keys (a share of a K/V head's) go to one XCD, one behind the other: ids go round over the 8 XCDs, and
    // the shares with them, a head's neighbours first.
    const int Hkv = a.kv.Hkv, n_groups = a.kv.batch * Hkv, i_xcd = blockIdx.x >> 3;
    const int unit = (blockIdx.x & 7) + 8 * (i_xcd / a.n_tiles), tile = i_xcd % a.n_tiles, split = unit / n_groups, group = unit - split * n_groups;
    if (split >= a.n_splits) return;
    const int b = group / Hkv, h = group - b * Hkv;
    const int Lc = min(max(a.ctx_len[b], 0), min(a.ctx_hint, a.kv.smax));
    const int nq = a.R * a.qpk;

    // queries: lane (g, c) holds, of query c of every tile, values VPL g + 8 s .. +8 of k-step s
    // (a query's row is worked out again where it is needed: kept through the loop it costs the registers that two tiles do not have)
    bf16x8 qf[U][KS];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int qc = min((tile * U + u) * 16 + c, nq - 1), row = qc / a.qpk, head = h * a.qpk + (qc - row * a.qpk);
        const uint16_t *src = a.q + (((int64_t)b * a.R + row) * (a.qpk * Hkv) + head) * HD + VPL * g;
#pragma unroll
        for (int s = 0; s < KS; s++) qf[u][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(src + 8 * s));
    }
    const int last_row = min((tile + 1) * U * 16 - 1, nq - 1) / a.qpk;          // of the workgroup: pass rows behind it are nobody's ancestors

    const int n_p = (a.P + AMX_CHUNK - 1) / AMX_CHUNK, n_c = (Lc + AMX_CHUNK - 1) / AMX_CHUNK, n_r = last_row / AMX_CHUNK + 1;
    const int n_chunks = n_p + n_c + n_r, per_split = (n_chunks + a.n_splits - 1) / a.n_splits;
    const int first = split * per_split + wave, end = min(n_chunks, (split + 1) * per_split);

    f32x4 o[U][NT];
    float m_run[U], base[U], l_run[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
#pragma unroll
        for (int n = 0; n < NT; n++) o[u][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run[u] = -INFINITY;
        base[u] = l_run[u] = 0.f;
    }
    unsigned char *v_lds = smem + wave * C::V_BYTES;
    // V row rho in LDS: 16-byte column p of it at position p ^ swizzle(rho)
    auto v_swizzle = [](int rho) __attribute__((always_inline)) { return HD == 128 ? 2 * (rho & 7) : 2 * ((rho >> 1) & 3); };

    auto load = [&](int chunk, Raw &r) __attribute__((always_inline)) {
        const int base_key = chunk * AMX_CHUNK;
#pragma unroll
        for (int tt = 0; tt < 2; tt++) {
            const int key = min(base_key + 16 * tt + c, Lc - 1);                // (behind the end: the last one once more, which has probability 0 there)
            const int64_t at = mx_row(a.kv, b, h, key);
            const int64_t byte = at * (HD * BITS / 8) + g * (DW * 4);
            const int64_t sc = at * (HD / 32) + (HD == 128 ? g : g >> 1);
#pragma unroll
            for (int d = 0; d < DW; d += (DW >= 4 ? 4 : 2)) {
                if constexpr (DW >= 4) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(a.kv.k + byte + 4 * d), y = *reinterpret_cast<const uint4 *>(a.kv.v + byte + 4 * d);
                    r.k[tt][d] = x.x; r.k[tt][d + 1] = x.y; r.k[tt][d + 2] = x.z; r.k[tt][d + 3] = x.w;
                    r.v[tt][d] = y.x; r.v[tt][d + 1] = y.y; r.v[tt][d + 2] = y.z; r.v[tt][d + 3] = y.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2 *>(a.kv.k + byte), y = *reinterpret_cast<const uint2 *>(a.kv.v + byte);
                    r.k[tt][0] = x.x; r.k[tt][1] = x.y;
                    r.v[tt][0] = y.x; r.v[tt][1] = y.y;
                }
            }
            r.ks[tt] = a.kv.k_scale[sc];
            r.vs[tt] = a.kv.v_scale[sc];
        }
    };
    auto decode = [&](const uint32_t (&d)[DW], float scale, bf16x8 (&x)[KS]) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < KS; s++) {
            if constexpr (BITS == 4) x[s] = mx_decode4(d[s], scale);
            else x[s] = mx_decode8(d[2 * s], d[2 * s + 1], scale);
        }
    };

    // V rows rho = 16 tt + c as bf16 to LDS
    auto put_v = [&](int tt, const bf16x8 (&vf)[KS]) __attribute__((always_inline)) {
        const int rho = 16 * tt + c;
#pragma unroll
        for (int s = 0; s < KS; s++)
            *reinterpret_cast<uint4 *>(v_lds + rho * (HD * 2) + (((KS * g + s) ^ v_swizzle(rho)) * 16)) = __builtin_bit_cast(uint4, vf[s]);
    };
    // V^T fragments: lane (g, c), tile n: column 16 n + c of keys 4g .. 4g+3 and 16 + 4g ..
    auto get_vt = [&](bf16x8 (&vt)[NT]) __attribute__((always_inline)) {
        typedef __attribute__((ext_vector_type(4))) short s4;
        typedef __attribute__((ext_vector_type(8))) short s8;
        typedef __attribute__((address_space(3))) s4 *lds_s4;
#pragma unroll
        for (int n = 0; n < NT; n++) {
            s4 half[2];
#pragma unroll
            for (int tt = 0; tt < 2; tt++) {
                const int rho = 16 * tt + 4 * g + (c >> 2);                     // lane (g, c) names row 4g + c/4, columns 4 (c % 4) ..
                half[tt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s4)(v_lds + rho * (HD * 2) + (((2 * n + ((c & 3) >> 1)) ^ v_swizzle(rho)) * 16) + (c & 1) * 8));
            }
            vt[n] = __builtin_bit_cast(bf16x8, s8{half[0][0], half[0][1], half[0][2], half[0][3], half[1][0], half[1][1], half[1][2], half[1][3]});
        }
    };
    auto scores = [&](int u, const bf16x8 (&kf)[2][KS], f32x4 (&sc)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int tt = 0; tt < 2; tt++) {
            sc[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; s++) sc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[tt][s], qf[u][s], sc[tt], 0, 0, 0);
        }
    };
    // scores of keys 4g + e, 16 + 4g + e (of which `bits` are seen) to probabilities; the running state of tile u moves on
    auto probabilities = [&](int u, const f32x4 (&sc)[2], uint32_t bits) __attribute__((always_inline)) -> bf16x8 {
        float s[8];
#pragma unroll
        for (int e = 0; e < 8; e++) s[e] = sc[e >> 2][e & 3] * a.scale_log2;
        if (__builtin_amdgcn_ballot_w64(bits != 0xFF) != 0) {
#pragma unroll
            for (int e = 0; e < 8; e++) s[e] = (bits >> e & 1) ? s[e] : -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int e = 1; e < 8; e++) mx = fmaxf(mx, s[e]);
        // the maximum moves rarely after the first chunks: only then are the lane groups compared and the sums rescaled
        if (__builtin_amdgcn_ballot_w64(mx > m_run[u]) != 0) {
            const float m_new = fmaxf(m_run[u], amx_over_groups(mx, [](float x, float y) { return fmaxf(x, y); }));
            base[u] = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = amx_exp2(m_run[u] - base[u]);
            m_run[u] = m_new;
            l_run[u] *= alpha;
#pragma unroll
            for (int n = 0; n < NT; n++) o[u][n] *= alpha;
        }
        uint32_t pk[4];
        float ps = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float p0 = amx_exp2(s[e] - base[u]), p1 = amx_exp2(s[e + 1] - base[u]);
            ps += p0 + p1;
            pk[e >> 1] = amx_pk_bf16(p0, p1);
        }
        l_run[u] += ps;
        return __builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3]));
    };

    // ---- the cache
    int chunk = first;
    {
        Raw raw;
        const int stop = min(end, n_c);
        if (chunk < stop) load(chunk, raw);
        for (; chunk < stop; chunk += W) {
            const int key0 = AMX_CHUNK * chunk;
            bf16x8 kf[2][KS];
#pragma unroll
            for (int tt = 0; tt < 2; tt++) {
                bf16x8 vf[KS];
                decode(raw.k[tt], mx_scale(raw.ks[tt]), kf[tt]);
                decode(raw.v[tt], mx_scale(raw.vs[tt]), vf);
                put_v(tt, vf);
            }
            if (chunk + W < stop) load(chunk + W, raw);
            f32x4 sc[U][2];
#pragma unroll
            for (int u = 0; u < U; u++) scores(u, kf, sc[u]);
            bf16x8 vt[NT];
            get_vt(vt);
            uint32_t bits = 0xFF;
            if (key0 + AMX_CHUNK > Lc) {
                bits = 0;
#pragma unroll
                for (int e = 0; e < 8; e++) bits |= (key0 + 16 * (e >> 2) + 4 * g + (e & 3) < Lc ? 1u : 0u) << e;
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                const bf16x8 pf = probabilities(u, sc[u], bits);
#pragma unroll
                for (int n = 0; n < NT; n++) o[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[n], pf, o[u][n], 0, 0, 0);
            }
        }
    }
    // ---- the prefix and the pass' rows: bf16, not seen by every query
    for (; chunk < end; chunk += W) {
        const bool in_prefix = chunk < n_c + n_p;
        const int key0 = AMX_CHUNK * (in_prefix ? chunk - n_c : chunk - n_c - n_p), n_keys = in_prefix ? a.P : a.R;
        bf16x8 kf[2][KS];
#pragma unroll
        for (int tt = 0; tt < 2; tt++) {
            const int key = min(key0 + 16 * tt + c, n_keys - 1);
            const int64_t off = ((int64_t)h * a.P + key) * HD;
            const uint16_t *ks = (in_prefix ? a.prompt_k + off : a.k_rows + a.k_at.at(b, h, key)) + VPL * g;
            const uint16_t *vs = (in_prefix ? a.prompt_v + off : a.v_rows + a.v_at.at(b, h, key)) + VPL * g;
            bf16x8 vf[KS];
#pragma unroll
            for (int s = 0; s < KS; s++) {
                kf[tt][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(ks + 8 * s));
                vf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(vs + 8 * s));
            }
            put_v(tt, vf);
        }
        bf16x8 vt[NT];
        get_vt(vt);
        bool odd = false;
#pragma unroll
        for (int n = 0; n < NT; n++) odd = odd || has_nonfinite(vt[n]);
        odd = __builtin_amdgcn_ballot_w64(odd) != 0;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int row = min((tile * U + u) * 16 + c, nq - 1) / a.qpk;
            const uint64_t sees = in_prefix ? (a.t.is_mask[row] ? ~0ull : 0) : a.t.anc[(int64_t)row * a.t.words + (key0 >> 6)] >> (key0 & 63);
            uint32_t bits = 0;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const int k = 16 * (e >> 2) + 4 * g + (e & 3);
                bits |= (key0 + k < n_keys && (sees >> k & 1) ? 1u : 0u) << e;
            }
            f32x4 sc[2];
            scores(u, kf, sc);
            const bf16x8 pf = probabilities(u, sc, bits);
            bf16x8 seen = {};                                                   // 1 where a key is seen
            if (odd) {
                uint32_t one[4];
#pragma unroll
                for (int e = 0; e < 4; e++) one[e] = (bits >> (2 * e) & 1 ? 0x3F80u : 0u) | (bits >> (2 * e) & 2 ? 0x3F800000u : 0u);
                seen = __builtin_bit_cast(bf16x8, make_uint4(one[0], one[1], one[2], one[3]));
            }
#pragma unroll
            for (int n = 0; n < NT; n++) {
                bf16x8 v = vt[n];
                if (odd) {                                                      // infinities or NaN among the rows
                    asm volatile("" : "+v"(v));                                 // (not worked out for all tiles ahead of time)
                    bf16x8 up, down;
                    split_nonfinite(v, up, down);
                    const f32x4 n_up = __builtin_amdgcn_mfma_f32_16x16x32_bf16(up, seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                    const f32x4 n_down = __builtin_amdgcn_mfma_f32_16x16x32_bf16(down, seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; r++) o[u][n][r] += nonfinite_term(n_up[r]) - nonfinite_term(n_down[r]);
                }
                o[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf, o[u][n], 0, 0, 0);
            }
        }
    }

    // ---- the waves' results meet: maxima and sums first, then the tiles, rescaled, summed in wave order
    float *sm = reinterpret_cast<float *>(smem + C::ML), *sl = sm + U * W * 16;         // [U][W][16]
    float4 *region = reinterpret_cast<float4 *>(smem);                                  // [U][W][NT][64]
#pragma unroll
    for (int u = 0; u < U; u++) {
        const float l = amx_over_groups(l_run[u], [](float x, float y) { return x + y; });
        if (g == 0) {
            sm[(u * W + wave) * 16 + c] = m_run[u];
            sl[(u * W + wave) * 16 + c] = l;
        }
    }
    __syncthreads();                                                                    // (and every wave is past its V region)
    float m_tot[U], l_tot[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        m_tot[u] = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; w++) m_tot[u] = fmaxf(m_tot[u], sm[(u * W + w) * 16 + c]);
        const float m_use = m_tot[u] == -INFINITY ? 0.f : m_tot[u];
        l_tot[u] = 0.f;
#pragma unroll
        for (int w = 0; w < W; w++) l_tot[u] += sl[(u * W + w) * 16 + c] * amx_exp2(sm[(u * W + w) * 16 + c] - m_use);
        const float f = amx_exp2(m_run[u] - m_use);
#pragma unroll
        for (int n = 0; n < NT; n++)
            region[((u * W + wave) * NT + n) * 64 + lane] = make_float4(o[u][n][0] * f, o[u][n][1] * f, o[u][n][2] * f, o[u][n][3] * f);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int qi = (tile * U + u) * 16 + c, row = qi / a.qpk;
        if (qi >= nq) continue;
        const bool absent = a.token && !a.t.is_mask[row] && a.token[(int64_t)b * a.R + row] < 0;
        const int64_t qrow = ((int64_t)b * a.R + row) * (a.qpk * Hkv) + h * a.qpk + (qi - row * a.qpk);
#pragma unroll
        for (int n = wave; n < NT; n += W) {
            float4 x = region[(u * W * NT + n) * 64 + lane];
#pragma unroll
            for (int w = 1; w < W; w++) {
                const float4 y = region[((u * W + w) * NT + n) * 64 + lane];
                x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
            }
            if (a.n_splits > 1) {
                *reinterpret_cast<float4 *>(a.part_o + (qrow * a.n_splits + split) * HD + 16 * n + 4 * g) = x;
                if (n == 0 && g == 0) *reinterpret_cast<float2 *>(a.part_ml + (qrow * a.n_splits + split) * 2) = make_float2(m_tot[u], absent ? 0.f : l_tot[u]);
                continue;
            }
            // (a NaN sum stays one; a sum of nothing, or an absent row, gives zeros)
            const float inv = absent || l_tot[u] == 0.f ? 0.f : 1.0f / l_tot[u];
            const uint2 w2 = absent ? make_uint2(0, 0) : make_uint2(amx_pk_bf16(x.x * inv, x.y * inv), amx_pk_bf16(x.z * inv, x.w * inv));
            *reinterpret_cast<uint2 *>(a.out + qrow * HD + 16 * n + 4 * g) = w2;
        }
    }
}

// o = sum_s w_s o_s / sum_s w_s l_s, w_s = 2^(m_s - max m); a thread 4 values of a query's head
template <int HD>
__global__ __launch_bounds__(256) void attn_mx_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml, int64_t n_queries, int n_splits,
                                                            uint16_t *__restrict__ out) {
    constexpr int LANES = HD / 4;
    const int64_t qrow = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int i = threadIdx.x % LANES * 4;
    if (qrow >= n_queries) return;
    const float2 *ml = reinterpret_cast<const float2 *>(part_ml) + qrow * n_splits;
    float m = -INFINITY;
    for (int s = 0; s < n_splits; s++) m = fmaxf(m, ml[s].x);
    const float m_use = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    bool absent = true;
    for (int s = 0; s < n_splits; s++) {
        const float w = amx_exp2(ml[s].x - m_use);
        const float4 o = *reinterpret_cast<const float4 *>(part_o + (qrow * n_splits + s) * HD + i);
        absent = absent && ml[s].y == 0.f;
        l += w * ml[s].y;
        x.x += w * o.x; x.y += w * o.y; x.z += w * o.z; x.w += w * o.w;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    *reinterpret_cast<uint2 *>(out + qrow * HD + i) = absent ? make_uint2(0, 0) : make_uint2(amx_pk_bf16(x.x * inv, x.y * inv), amx_pk_bf16(x.z * inv, x.w * inv));
}

struct AmxPlan { int tiles_u, n_tiles, splits; int64_t workgroups; size_t part_o, part_ml; };

// Queries in tiles of 16, two of them a workgroup where there are two; the keys split until the chip is full or a wave has a chunk or two.
static AmxPlan amx_plan(int batch, int rows, int Hq, int Hkv, int hd, int ctx_hint, int n_prompt) {
    AmxPlan p;
    const int64_t nq = (int64_t)rows * (Hq / Hkv);
    p.tiles_u = nq > 16 ? 2 : 1;
    p.n_tiles = (int)((nq + 16 * p.tiles_u - 1) / (16 * p.tiles_u));
    const int64_t chunks = ((int64_t)n_prompt + AMX_CHUNK - 1) / AMX_CHUNK + ((int64_t)ctx_hint + AMX_CHUNK - 1) / AMX_CHUNK + (rows + AMX_CHUNK - 1) / AMX_CHUNK;
    const int64_t wgs = (int64_t)batch * Hkv * p.n_tiles;
    int64_t splits = (512 + wgs - 1) / wgs, most = (chunks + 2 * AMX_WAVES - 1) / (2 * AMX_WAVES);
    if (splits > most) splits = most;
    if (splits > 256) splits = 256;
    if (splits < 1) splits = 1;
    p.splits = (int)splits;
    p.workgroups = wgs * splits;
    const size_t queries = (size_t)batch * rows * Hq;
    p.part_o = splits > 1 ? (queries * splits * hd * 4 + 255) / 256 * 256 : 0;
    p.part_ml = splits > 1 ? (queries * splits * 8 + 255) / 256 * 256 : 0;
    return p;
}

static int amx_sizes(const char *who, int32_t batch, int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t bits, int32_t ctx_hint, int32_t n_prompt) {
    if (batch <= 0 || rows <= 0 || rows > BITA_MAX_ROWS || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads || ctx_hint < 0 || n_prompt < 0)
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: non-positive or inconsistent size", who);
    if ((head_dim != 64 && head_dim != 128) || (bits != 4 && bits != 8)) return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: head_dim 64 or 128, bits 4 or 8", who);
    if (ctx_hint > (1 << 30) || n_prompt > (1 << 20) || (int64_t)batch * n_heads > (1 << 17))
        return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: at most 2^30 slots, 2^20 prefix rows, 2^17 sequences times heads", who);
    return BITA_OK;
}

extern "C" size_t bita_tree_attention_mx_workspace_bytes(int32_t batch, int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t bits,
                                                         int32_t ctx_hint, int32_t n_prompt) {
    if (amx_sizes("bita_tree_attention_mx_workspace_bytes", batch, rows, n_heads, n_kv_heads, head_dim, bits, ctx_hint, n_prompt)) return 0;
    const AmxPlan p = amx_plan(batch, rows, n_heads, n_kv_heads, head_dim, ctx_hint, n_prompt);
    return p.part_o + p.part_ml;
}

extern "C" int bita_tree_attention_mx_plan_info(int32_t batch, int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t bits, int32_t ctx_hint,
                                                int32_t n_prompt, int32_t *out4) {
    if (!out4) return bita_set_error(BITA_ERR_INVALID_ARG, "bita_tree_attention_mx_plan_info: null argument");
    if (int rc = amx_sizes("bita_tree_attention_mx_plan_info", batch, rows, n_heads, n_kv_heads, head_dim, bits, ctx_hint, n_prompt)) return rc;
    const AmxPlan p = amx_plan(batch, rows, n_heads, n_kv_heads, head_dim, ctx_hint, n_prompt);
    out4[0] = p.splits; out4[1] = 16 * p.tiles_u; out4[2] = AMX_WAVES;
    out4[3] = p.workgroups < INT32_MAX ? (int32_t)p.workgroups : INT32_MAX;
    return BITA_OK;
}

template <int HD, int BITS, int U>
static void launch_amx(const AmxArgs &a, int64_t n_groups, hipStream_t s) {
    static_assert(AmxCfg<HD, U>::SMEM <= 80 * 1024, "two workgroups a CU");
    (void)hipFuncSetAttribute((const void *)attn_mx_kernel<HD, BITS, U>, hipFuncAttributeMaxDynamicSharedMemorySize, AmxCfg<HD, U>::SMEM);
    const dim3 grid((unsigned)((n_groups * a.n_splits + 7) / 8 * 8 * a.n_tiles));
    hipLaunchKernelGGL((attn_mx_kernel<HD, BITS, U>), grid, dim3(AMX_WAVES * 64), (AmxCfg<HD, U>::SMEM), s, a);
}

extern "C" int bita_tree_attention_mx(const bita_tree_template *t, const void *d_q, const bita_kv_mx *kv, const void *d_k_rows, int64_t k_seq, int64_t k_head,
                                      int64_t k_row, const void *d_v_rows, int64_t v_seq, int64_t v_head, int64_t v_row, const void *d_prompt_k, const void *d_prompt_v,
                                      int32_t n_prompt, const int32_t *d_ctx_len, const int32_t *d_token, int32_t n_heads, int32_t ctx_hint, void *d_ws,
                                      size_t ws_bytes, void *d_out, void *stream) {
    const char *who = "bita_tree_attention_mx";
    if (!t || !d_q || !kv || !d_k_rows || !d_v_rows || !d_ctx_len || !d_out || (n_prompt > 0 && (!d_prompt_k || !d_prompt_v)))
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: null argument", who);
    AmxArgs a;
    if (int rc = kv_mx_of(kv, &a.kv, who)) return rc;
    if (int rc = amx_sizes(who, kv->batch, t->dev.rows, n_heads, kv->n_kv_heads, kv->head_dim, kv->bits, ctx_hint, n_prompt)) return rc;
    if (ctx_hint > kv->smax) return bita_set_error(BITA_ERR_CAPACITY, "%s: ctx_hint %d outside capacity %d", who, ctx_hint, kv->smax);
    a.k_at = MxRows{k_seq, k_head, k_row};
    a.v_at = MxRows{v_seq, v_head, v_row};
    if (int rc = mx_rows_check(who, a.k_at, a.v_at, (uintptr_t)d_q | (uintptr_t)d_k_rows | (uintptr_t)d_v_rows | (uintptr_t)d_prompt_k | (uintptr_t)d_prompt_v |
                                                        (uintptr_t)d_out | (uintptr_t)d_ws)) return rc;
    const AmxPlan p = amx_plan(kv->batch, t->dev.rows, n_heads, kv->n_kv_heads, kv->head_dim, ctx_hint, n_prompt);
    if (ws_bytes < p.part_o + p.part_ml || (p.splits > 1 && !d_ws))
        return bita_set_error(BITA_ERR_CAPACITY, "%s: workspace %zu < %zu bytes", who, ws_bytes, p.part_o + p.part_ml);
    a.t = t->dev;
    a.q = (const uint16_t *)d_q; a.k_rows = (const uint16_t *)d_k_rows; a.v_rows = (const uint16_t *)d_v_rows;
    a.prompt_k = (const uint16_t *)d_prompt_k; a.prompt_v = (const uint16_t *)d_prompt_v;
    a.ctx_len = d_ctx_len; a.token = d_token;
    a.P = n_prompt; a.R = t->dev.rows; a.qpk = n_heads / kv->n_kv_heads; a.ctx_hint = ctx_hint;
    a.n_tiles = p.n_tiles; a.n_splits = p.splits;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)kv->head_dim);
    a.part_o = (float *)d_ws; a.part_ml = (float *)((unsigned char *)d_ws + p.part_o);
    a.out = (uint16_t *)d_out;
    hipStream_t s = (hipStream_t)stream;
    const int64_t groups = (int64_t)kv->batch * kv->n_kv_heads;
#define AMX_LAUNCH(HD_, BITS_) do { if (p.tiles_u == 2) launch_amx<HD_, BITS_, 2>(a, groups, s); else launch_amx<HD_, BITS_, 1>(a, groups, s); } while (0)
    if (kv->head_dim == 128) { if (kv->bits == 4) AMX_LAUNCH(128, 4); else AMX_LAUNCH(128, 8); }
    else { if (kv->bits == 4) AMX_LAUNCH(64, 4); else AMX_LAUNCH(64, 8); }
#undef AMX_LAUNCH
    if (p.splits > 1) {
        const int64_t queries = (int64_t)kv->batch * t->dev.rows * n_heads;
        const int per_wg = 1024 / kv->head_dim;
        const dim3 grid((unsigned)((queries + per_wg - 1) / per_wg));
        if (kv->head_dim == 128) hipLaunchKernelGGL((attn_mx_merge_kernel<128>), grid, dim3(256), 0, s, a.part_o, a.part_ml, queries, p.splits, a.out);
        else hipLaunchKernelGGL((attn_mx_merge_kernel<64>), grid, dim3(256), 0, s, a.part_o, a.part_ml, queries, p.splits, a.out);
    }
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}
