// Attention of a pass' rows over a K/V cache in 4 or 8 bits: o = softmax(q k^T / sqrt(d)) v over [prefix | cache | pass rows], the
// prefix seen by mask rows, the pass rows by their descendants-or-self.
//
// A K/V head's queries are one axis: R rows times the heads of its group, 16 of them a tile, whatever the number of heads.  A workgroup
// owns U tiles and a share of the keys, which its waves walk in chunks of 32, each with its own running maximum and sum; the waves' results meet
// in LDS once at the end, the shares' (where the keys are split over workgroups) in a second kernel.
//  * Codes go from memory to registers, two chunks ahead of the arithmetic (one with two tiles), and from there to bf16 (exact: a code times a power of two) by
//    conversion instructions that apply the scale: a lane holds a quarter of a key's head, one block of 32 values (half of one at 64).
//  * The contraction over the head runs in the order in which a lane holds it: k-step s takes values 8s .. 8s+7 of every lane's
//    quarter, of the queries too, so K needs no other layout than the cache's.
//  * S^T = K Q^T leaves lane (g, c) the scores of keys 4g .. 4g+3 of either half of the chunk for query c, which is the
//    B operand of O^T = V^T P^T if that product takes the keys in the same order: probabilities stay in registers.
//  * V^T needs eight keys of one column in a lane: V goes to LDS as bf16 rows and comes back by transposed reads.  The region is the wave's own,
//    and its LDS instructions run in order, so there is no barrier in the loop.
// Bound by what a CU takes in at low batch (one sequence of 131072 keys, 64/8 heads, 4 bits: 143 MB in 27 us, 5.3 TB/s, and a merge of 4), by its own start and end at
// short lengths (1000 keys, 32 heads: 10 us for 4.4 MB), by the conversions and the exponentials between, where a K/V head has many queries by matrix instructions.
#include <algorithm>
#include <climits>
#include <cmath>
#include "mx.h"
#include "attention_core.h"

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
    int P, R, qpk, ctx_hint, n_tiles, n_shares, per_share;      // tiles of a workgroup's queries; shares of all sequences' keys together (as many: nothing is split); turns of a share where the batch is large
    float scale_log2;
    float *part_o, *part_ml;                                    // [share][R * heads][HD], [..][2]
    int2 *share_of;                                             // [batch]: a sequence's first share and how many it has (one: the result is in out)
    uint16_t *out;
    __device__ __forceinline__ int length(int b) const { return min(max(ctx_len[b], 0), min(ctx_hint, kv.smax)); }
    // of a query (row, head) of sequence b: where it is in out and q, and where in a share's part
    __device__ __forceinline__ int64_t query(int b, int row, int head) const { return ((int64_t)b * R + row) * (qpk * kv.Hkv) + head; }
    __device__ __forceinline__ int64_t part(int share, int row, int head) const { return ((int64_t)share * R + row) * (qpk * kv.Hkv) + head; }
};

__device__ __forceinline__ uint32_t amx_sum(uint32_t x) {                       // over the wave: rows of 16 lanes by rotation, then the four rows
    x += __builtin_amdgcn_update_dpp(0, x, 0x121, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x122, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x124, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, false);
    return __builtin_amdgcn_readlane(x, 0) + __builtin_amdgcn_readlane(x, 16) + __builtin_amdgcn_readlane(x, 32) + __builtin_amdgcn_readlane(x, 48);
}
__device__ __forceinline__ uint32_t amx_running_sum(uint32_t x, int lane) {     // of this lane and those before it
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);             // (row_shr 1, 2, 4, 8: 0 comes in)
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    const uint32_t r0 = __builtin_amdgcn_readlane(x, 15), r1 = r0 + __builtin_amdgcn_readlane(x, 31), r2 = r1 + __builtin_amdgcn_readlane(x, 47);
    return x + (lane < 16 ? 0 : lane < 32 ? r0 : lane < 48 ? r1 : r2);
}

// What a workgroup does: a tile of queries of K/V head h of sequence b, over chunks first .. end of its keys (the cache's, the prefix', the pass rows'; KEYS a chunk, TURN
// chunks at a time), which are one share of all.
//
// The shares are cut from the lengths that are there, not from the hint: of all sequences together as many as the host has workgroups for, none longer than it has
// to be.  With c_b turns in sequence b, p of them a share, there are sum ceil(c_b / p) <= T / p + batch (1 - 1 / p) shares, T = sum c_b: p is at
// least T / shares, and T / (shares - batch + 1) is enough; between the two every wave looks for the smallest that fits, the sequences in its lanes.  A batch of more than
// a wave's lanes is cut by the hint: it has workgroups enough.
struct AmxPlace { int tile, share, b, h, first, end, length; bool split; };  // split: the sequence has other shares
// The arguments for a kernel's end, read again there: kept through the loops, scalar registers spilled.
__device__ __forceinline__ AmxArgs amx_again() {
    auto p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    AmxArgs a;
    __builtin_memcpy(&a, (const void *)p, sizeof a);
    return a;
}
template <int KEYS, int TURN>
__device__ __forceinline__ bool amx_place(const AmxArgs &a, AmxPlace &w) {
    // The tiles that read the same keys go to one XCD, one behind the other: ids go round over the 8 XCDs.  (Quotients are worked out in vector registers: without
    // being told, the compiler keeps what follows from them there, descriptors too.)
    const int i = blockIdx.x >> 3, set = __builtin_amdgcn_readfirstlane(i / a.n_tiles), unit = (blockIdx.x & 7) + 8 * set;
    w.tile = __builtin_amdgcn_readfirstlane(i - set * a.n_tiles);
    w.share = __builtin_amdgcn_readfirstlane(unit / a.kv.Hkv);
    w.h = __builtin_amdgcn_readfirstlane(unit - w.share * a.kv.Hkv);
    if (w.share >= a.n_shares) return false;
    const int batch = a.kv.batch, more = (a.P + KEYS - 1) / KEYS + (a.R - 1) / KEYS + 1, lane = threadIdx.x & 63;
    auto turns = [&](int n) __attribute__((always_inline)) { return (uint32_t)((n + KEYS - 1) / KEYS + more + TURN - 1) / TURN; };
    uint32_t per, mine, count, at;
    if (a.n_shares == batch) {
        w.b = w.share;
        w.length = __builtin_amdgcn_readfirstlane(a.length(w.b));
        w.first = 0;
        w.end = INT_MAX;
        w.split = false;
        return true;
    }
    if (batch > 64) {
        mine = __builtin_amdgcn_readfirstlane(w.share / batch);
        w.b = at = w.share - mine * batch;
        w.length = __builtin_amdgcn_readfirstlane(a.length(w.b));
        per = a.per_share;
        count = __builtin_amdgcn_readfirstlane((turns(w.length) + per - 1) / per);
        if (mine >= count) return false;
    } else {
        const int len = lane < batch ? a.length(lane) : 0;
        const uint32_t c = lane < batch ? turns(len) : 0, all = amx_sum(c), shares = a.n_shares;
        per = __builtin_amdgcn_readfirstlane((all + shares - 1) / shares);
        uint32_t enough = __builtin_amdgcn_readfirstlane((all + shares - batch) / (shares - batch + 1));
        while (per < enough) {
            const uint32_t p = (per + enough) / 2;
            if (amx_sum((c + p - 1) / p) <= shares) enough = p;
            else per = p + 1;
        }
        const uint32_t n = (c + per - 1) / per, behind = amx_running_sum(n, lane);
        const uint64_t later = __builtin_amdgcn_ballot_w64(behind > (uint32_t)w.share);
        if (later == 0) return false;
        w.b = __builtin_ctzll(later);
        count = __builtin_amdgcn_readlane(n, w.b);
        at = __builtin_amdgcn_readlane(behind, w.b) - count;
        mine = w.share - at;
        w.length = __builtin_amdgcn_readlane(len, w.b);
    }
    w.b = __builtin_amdgcn_readfirstlane(w.b);
    w.length = __builtin_amdgcn_readfirstlane(w.length);
    w.first = __builtin_amdgcn_readfirstlane(mine * per * TURN);
    w.end = __builtin_amdgcn_readfirstlane(w.first + per * TURN);
    w.split = __builtin_amdgcn_readfirstlane(count) > 1;
    if (mine == 0 && w.h == 0 && w.tile == 0 && threadIdx.x == 0) a.share_of[w.b] = make_int2(at, count);
    return true;
}

// Sixteen neighbouring keys' codes and scale bytes, from one page or the contiguous cache: lane (g, c) = (l / 16, l % 16) takes a quarter of key c,
// HD / 4 values.  The keys' first row is known to the whole wave, so a descriptor holds it, with the keys that there are (none: what
// is loaded is 0, which decodes to 0), and a lane's own offsets never change.
template <int HD, int BITS>
struct MxKeys {
    static constexpr int DW = HD / 4 * BITS / 32, ROW = HD * BITS / 8, SROW = HD / 32;      // dwords of a lane, bytes of a row's codes, and of its scales
    static constexpr int PARTS = HD / 32;                                                   // eights of values of a lane
    uint32_t d[DW], scale;

    static __device__ __forceinline__ uint32_t code_offset(int lane) { return (lane & 15) * ROW + (lane >> 4) * (DW * 4); }
    static __device__ __forceinline__ uint32_t scale_offset(int lane) { return (lane & 15) * SROW + (HD == 128 ? lane >> 4 : lane >> 5); }
    // the page of keys key0 .. key0 + 15 of sequence b, of which there are `length` (a number the whole wave has)
    static __device__ __forceinline__ int page_of(const KvMx &kv, int b, int key0, int length) {
        if (!kv.table) return b;
        const int32_t *at = kv.table + (int64_t)b * kv.max_pages + (min(key0, length - 1) >> kv.page_lg);
        return __builtin_amdgcn_readfirstlane(min(max(*(const __attribute__((address_space(4))) int32_t *)(uintptr_t)at, 0), kv.n_pages - 1));      // (through the scalar cache)
    }
    __device__ __forceinline__ void load(const KvMx &kv, const unsigned char *codes, const uint8_t *scales, int h, int key0, int length, int page,
                                         uint32_t code_off, uint32_t scale_off) {
        const int64_t row = ((int64_t)page * kv.Hkv + h) * kv.page_rows + (key0 & kv.slot_mask);
        const int n = __builtin_amdgcn_readfirstlane(min(max(length - key0, 0), 16));       // (limits are taken in vector registers, and the descriptor with them)
        take(__builtin_amdgcn_make_buffer_rsrc((void *)(codes + row * ROW), 0, n * ROW, 0x00027000),
             __builtin_amdgcn_make_buffer_rsrc((void *)(scales + row * SROW), 0, n * SROW, 0x00027000), code_off, scale_off);
    }
    __device__ __forceinline__ void take(__amdgpu_buffer_rsrc_t rc, __amdgpu_buffer_rsrc_t rs, uint32_t code_off, uint32_t scale_off) {
        if constexpr (DW == 2) {
            typedef __attribute__((ext_vector_type(2))) uint32_t u2;
            const u2 v = __builtin_amdgcn_raw_buffer_load_b64(rc, code_off, 0, 0);
            d[0] = v[0]; d[1] = v[1];
        } else {
#pragma unroll
            for (int i = 0; i < DW; i += 4) {
                const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(rc, code_off + 4 * i, 0, 0);
                d[i] = v[0]; d[i + 1] = v[1]; d[i + 2] = v[2]; d[i + 3] = v[3];
            }
        }
        scale = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(rs, scale_off, 0, 0);
    }
    __device__ __forceinline__ void decode(bf16x8 (&x)[PARTS]) const {
        const float s = mx_scale(scale);
#pragma unroll
        for (int i = 0; i < PARTS; i++) {
            if constexpr (BITS == 4) x[i] = mx_decode4(d[i], s);
            else x[i] = mx_decode8(d[2 * i], d[2 * i + 1], s);
        }
    }
};

template <int HD, int U, int W>
struct AmxCfg {
    static constexpr int KS = HD / 32, NT = HD / 16, VPL = HD / 4;      // k-steps, 16-wide tiles of the head, values a lane holds of a key
    static constexpr int V_BYTES = AMX_CHUNK * HD * 2;                  // a wave's V chunk as bf16
    static constexpr int MERGE = U * W * NT * 64 * 16;
    static constexpr int ML = W * V_BYTES > MERGE ? W * V_BYTES : MERGE;
    static constexpr int SMEM = ML + 2 * U * W * 16 * 4;
};

template <int HD, int BITS, int U, int W>
__global__ __launch_bounds__(W * 64, 2) void attn_mx_kernel(AmxArgs a) {
    using C = AmxCfg<HD, U, W>;
    using Keys = MxKeys<HD, BITS>;
    constexpr int KS = C::KS, NT = C::NT, VPL = C::VPL;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    AmxPlace at;
    if (!amx_place<AMX_CHUNK, W>(a, at)) return;
    const int tile = at.tile, b = at.b, h = at.h, Lc = at.length, nq = a.R * a.qpk;

    // queries: lane (g, c) holds, of query c of every tile, values VPL g + 8 s .. +8 of k-step s
    // (a query's row is worked out again where it is needed: kept through the loop it costs the registers that two tiles do not have)
    bf16x8 qf[U][KS];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int qc = min((tile * U + u) * 16 + c, nq - 1), row = qc / a.qpk, head = h * a.qpk + (qc - row * a.qpk);
        const uint16_t *src = a.q + a.query(b, row, head) * HD + VPL * g;
#pragma unroll
        for (int s = 0; s < KS; s++) qf[u][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(src + 8 * s));
    }
    const int last_row = min((tile + 1) * U * 16 - 1, nq - 1) / a.qpk;          // of the workgroup: pass rows behind it are nobody's ancestors

    const int n_p = (a.P + AMX_CHUNK - 1) / AMX_CHUNK, n_c = (Lc + AMX_CHUNK - 1) / AMX_CHUNK, n_r = last_row / AMX_CHUNK + 1;
    const int first = at.first + wave, end = min(n_c + n_p + n_r, at.end);

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
        // Two chunks' codes are on their way while a third is multiplied: a chunk's arithmetic is shorter than a trip to memory under load.  (One, where
        // two tiles of queries make it longer and leave no registers.)
        constexpr int DEPTH = U == 1 ? 2 : 1;
        struct Chunk { Keys k[2], v[2]; int page[2]; };                         // of keys c and 16 + c; the pages to load from next
        Chunk set[DEPTH] = {};
        const uint32_t code_off = Keys::code_offset(lane), scale_off = Keys::scale_offset(lane);
        const int stop = min(end, n_c);
        const bool apart = a.kv.table && a.kv.page_rows < AMX_CHUNK;            // a chunk's halves lie in two pages
        auto ask_pages = [&](Chunk &x, int chunk) __attribute__((always_inline)) {
            x.page[0] = Keys::page_of(a.kv, b, AMX_CHUNK * chunk, Lc);
            if (apart) x.page[1] = Keys::page_of(a.kv, b, AMX_CHUNK * chunk + 16, Lc);
        };
        auto load = [&](Chunk &x, int chunk) __attribute__((always_inline)) {   // (behind the end: nothing is there, zeros come back)
            if (!apart) {                                                       // (half the descriptors: one token over 1000 keys 10.2 -> 9.8 us back to back, over 131072, sum included, 31.9 -> 31.0)
                const int key0 = AMX_CHUNK * chunk, n = __builtin_amdgcn_readfirstlane(min(max(Lc - key0, 0), AMX_CHUNK));
                const int64_t row = ((int64_t)x.page[0] * a.kv.Hkv + h) * a.kv.page_rows + (key0 & a.kv.slot_mask);
                auto two = [&](Keys (&y)[2], const unsigned char *codes, const uint8_t *scales) __attribute__((always_inline)) {
                    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc((void *)(codes + row * Keys::ROW), 0, n * Keys::ROW, 0x00027000);
                    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)(scales + row * Keys::SROW), 0, n * Keys::SROW, 0x00027000);
                    y[0].take(rc, rs, code_off, scale_off);
                    y[1].take(rc, rs, code_off + 16 * Keys::ROW, scale_off + 16 * Keys::SROW);
                };
                two(x.k, a.kv.k, a.kv.k_scale);
                two(x.v, a.kv.v, a.kv.v_scale);
                return;
            }
#pragma unroll
            for (int tt = 0; tt < 2; tt++) {
                x.k[tt].load(a.kv, a.kv.k, a.kv.k_scale, h, AMX_CHUNK * chunk + 16 * tt, Lc, x.page[tt], code_off, scale_off);
                x.v[tt].load(a.kv, a.kv.v, a.kv.v_scale, h, AMX_CHUNK * chunk + 16 * tt, Lc, x.page[tt], code_off, scale_off);
            }
        };
        auto step = [&](Chunk &x) __attribute__((always_inline)) {
            const int key0 = AMX_CHUNK * chunk;
            bf16x8 kf[2][KS];
#pragma unroll
            for (int tt = 0; tt < 2; tt++) {
                bf16x8 vf[KS];
                x.k[tt].decode(kf[tt]);
                x.v[tt].decode(vf);
                put_v(tt, vf);
            }
            load(x, chunk + DEPTH * W);
            ask_pages(x, chunk + 2 * DEPTH * W);
            f32x4 sc[U][2];
#pragma unroll
            for (int u = 0; u < U; u++) scores(u, kf, sc[u]);
            __builtin_amdgcn_sched_barrier(0);                                  // (K's registers are V's from here on)
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
            chunk += W;
        };
        if (chunk < stop) {
#pragma unroll
            for (int i = 0; i < DEPTH; i++) {
                ask_pages(set[i], chunk + i * W);
                load(set[i], chunk + i * W);
                ask_pages(set[i], chunk + (i + DEPTH) * W);
            }
            while (true) {
                step(set[0]);
                if (chunk >= stop) break;
                if constexpr (DEPTH > 1) {
                    step(set[1]);
                    if (chunk >= stop) break;
                }
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
    const AmxArgs z = amx_again();
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int qi = (tile * U + u) * 16 + c, row = qi / z.qpk;
        if (qi >= nq) continue;
        const bool absent = z.token && !z.t.is_mask[row] && z.token[(int64_t)b * z.R + row] < 0;
        const int head = h * z.qpk + (qi - row * z.qpk);
#pragma unroll
        for (int n = wave; n < NT; n += W) {
            float4 x = region[(u * W * NT + n) * 64 + lane];
#pragma unroll
            for (int w = 1; w < W; w++) {
                const float4 y = region[((u * W + w) * NT + n) * 64 + lane];
                x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
            }
            if (at.split) {
                const int64_t to = z.part(at.share, row, head);
                *reinterpret_cast<float4 *>(z.part_o + to * HD + 16 * n + 4 * g) = x;
                // (-inf says that there was nothing to sum: where no score was a number the sum is NaN and its reference any number, so that the sum over shares has it)
                const float ref = absent ? -INFINITY : m_tot[u] == -INFINITY && l_tot[u] != 0.f ? 0.f : m_tot[u];
                if (n == 0 && g == 0) *reinterpret_cast<float2 *>(z.part_ml + to * 2) = make_float2(ref, absent ? 0.f : l_tot[u]);
                continue;
            }
            // (a NaN sum stays one; a sum of nothing, or an absent row, gives zeros)
            const float inv = absent || l_tot[u] == 0.f ? 0.f : 1.0f / l_tot[u];
            const uint2 w2 = absent ? make_uint2(0, 0) : make_uint2(amx_pk_bf16(x.x * inv, x.y * inv), amx_pk_bf16(x.z * inv, x.w * inv));
            *reinterpret_cast<uint2 *>(z.out + z.query(b, row, head) * HD + 16 * n + 4 * g) = w2;
        }
    }
}

// Many queries a K/V head (a tree under grouped heads): a workgroup's waves own 32 queries each and share the keys, in tiles of 64 that they decode
// together into LDS, each wave 16 rows, a tile ahead of the products (attention_core.h).  Scores run a tile ahead of the values too, so
// K is decoded two tiles ahead and V one, from codes that were asked for a tile earlier.  A wave finishes its own queries.  Bound by exponentials, conversions and
// matrix instructions together: a turn of two workgroups on a CU is 2.1 us, 1020 TFLOP/s over the card (with one 1.37); four trees of 68 rows over 1024 to 4096 keys of 8 bits, 64/8
// heads, 50.6 us, and 6.3 for the shares' sum.
#define AMW_ROWS (32 * AMX_WAVES)

template <int HD, int BITS>
__global__ __launch_bounds__(AMX_WAVES * 64, 2) void attn_mx_wide_kernel(AmxArgs a) {
    using Core = AttnCore<HD>;
    using Keys = MxKeys<HD, BITS>;
    constexpr int TILE = Core::TILE, VPL = HD / 4, PARTS = Keys::PARTS;         // values a lane holds of a row: PARTS columns of 8
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];      // K tiles [2], V tiles [2]
    const int lane = threadIdx.x & 63, hf = lane >> 5, g16 = lane >> 4, c16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    AmxPlace at;
    if (!amx_place<CORE_KEYS, 1>(a, at)) return;
    const int tile = at.tile, b = at.b, h = at.h, Lc = at.length;
    const int nq = a.R * a.qpk;
    const bool idle = tile * AMW_ROWS + wave * 32 >= nq;                        // (it decodes all the same)
    // (what a lane is for, a query's row and its offsets, is worked out where it is used: kept through the loop, 8 bits of 128 spilled)
    auto query_now = [&]() __attribute__((always_inline)) { return min(tile * AMW_ROWS + wave * 32 + (core_lane() & 31), nq - 1); };

    Core core;
    core.init(lane);
    const int q_first = query_now(), q_at = q_first / a.qpk;
    const uint16_t *q_row = a.q + a.query(b, q_at, h * a.qpk + (q_first - q_at * a.qpk)) * HD;
#pragma unroll
    for (int s = 0; s < Core::KS; s++) core.q[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(q_row + 16 * s + 8 * hf));

    const int last_row = min((tile + 1) * AMW_ROWS - 1, nq - 1) / a.qpk;        // of the workgroup: pass rows behind it are nobody's ancestors
    const int n_c = (Lc + CORE_KEYS - 1) / CORE_KEYS, n_p = (a.P + CORE_KEYS - 1) / CORE_KEYS, n_all = n_c + n_p + last_row / CORE_KEYS + 1;
    const int begin = at.first, end = min(n_all, at.end), c_end = min(end, n_c);

    const uint32_t lds = (uint32_t)(size_t)((__attribute__((address_space(3))) unsigned char *)smem);
    auto k_tile = [&](int t) __attribute__((always_inline)) { return lds + (t & 1) * TILE; };
    auto v_tile = [&](int t) __attribute__((always_inline)) { return lds + 2 * TILE + (t & 1) * TILE; };
    auto meet = [&]() __attribute__((always_inline)) {                          // what was written to LDS can be read, what was read can be written over
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // This lane decodes row 16 wave + c16 of a tile, values VPL g16 ..: where they go
    const int my = 16 * wave + c16;
    uint32_t k_put = my * Core::ROW + (((PARTS * g16) ^ Core::k_swizzle(my)) * 16), v_put = my * Core::ROW + (((PARTS * g16) ^ Core::v_swizzle(my)) * 16);
    auto put = [&](uint32_t tile, bool is_v, const bf16x8 (&x)[PARTS]) __attribute__((always_inline)) {
        uint32_t at = tile + (is_v ? v_put : k_put);                            // (a lane's columns sit in address bits that the swizzle shares by exclusive or)
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int s = 0; s < PARTS; s++) *(__attribute__((address_space(3))) u32x4_t *)(uintptr_t)(at ^ (16 * s)) = __builtin_bit_cast(u32x4_t, x[s]);
    };
    auto first_key = [&](int t) __attribute__((always_inline)) { return t * CORE_KEYS + 16 * wave; };
    auto load_k = [&](int t, int page, Keys &x) __attribute__((always_inline)) { x.load(a.kv, a.kv.k, a.kv.k_scale, h, first_key(t), Lc, page, Keys::code_offset(core_lane()), Keys::scale_offset(core_lane())); };
    auto load_v = [&](int t, int page, Keys &x) __attribute__((always_inline)) { x.load(a.kv, a.kv.v, a.kv.v_scale, h, first_key(t), Lc, page, Keys::code_offset(core_lane()), Keys::scale_offset(core_lane())); };
    auto page_of = [&](int t) __attribute__((always_inline)) { return Keys::page_of(a.kv, b, first_key(t), Lc); };
    auto decode = [&](const Keys &x, uint32_t tile, bool is_v) __attribute__((always_inline)) {
        bf16x8 v[PARTS];
        x.decode(v);
        put(tile, is_v, v);
    };
    auto decode_k = [&](const Keys &x, int t) __attribute__((always_inline)) { decode(x, k_tile(t), false); };
    auto decode_v = [&](const Keys &x, int t) __attribute__((always_inline)) { decode(x, v_tile(t), true); };
    // scores of keys that `sees` has no bit for: none
    auto mask = [&](f32x16 (&s)[2], uint64_t sees) __attribute__((always_inline)) {
        sees >>= 4 * (core_lane() >> 5);
#pragma unroll
        for (int e = 0; e < 32; e++) {
            const uint32_t w = (uint32_t)(sees >> (e & 16 ? 32 : 0));
            s[e >> 4][e & 15] = w >> (8 * ((e & 15) >> 2) + (e & 3)) & 1 ? s[e >> 4][e & 15] : -INFINITY;
        }
    };
    auto up_to = [](int n) __attribute__((always_inline)) { return n >= 64 ? ~0ull : (1ull << n) - 1; };

    f32x16 s[2];
    uint32_t p[16], odd = 0;
    int t = begin;
    if (t < c_end) {
        Keys kc, vc;
        int page = page_of(t), page_next = page_of(t + 1);                      // of the tile whose V, and K, is loaded next
        load_k(t, page, kc);
        load_v(t, page, vc);
        decode_k(kc, t);
        load_k(t + 1, page_next, kc);                                           // (from here on possibly behind the share's end: never used there)
        meet();
        if (!idle) {
            core.scores(k_tile(t), s);
            if (t + 1 == n_c) mask(s, up_to(Lc - t * CORE_KEYS));
            core.take_maximum(core.largest(s), a.scale_log2);                   // (what every query's reference starts with)
        }
        page = page_next;
        page_next = page_of(t + 2);
        decode_v(vc, t);
        decode_k(kc, t + 1);
        load_v(t + 1, page, vc);
        load_k(t + 2, page_next, kc);
        auto turn = [&](int t, f32x16 (&now)[2], f32x16 (&next)[2]) __attribute__((always_inline)) {
            meet();                                                             // V of tile t and K of t + 1 are there
            page = page_next;
            page_next = page_of(t + 3);
            decode_v(vc, t + 1);
            decode_k(kc, t + 2);
            load_v(t + 2, page, vc);
            load_k(t + 3, page_next, kc);
            if (idle) return;
            core.scores_and_probabilities(k_tile(t + 1), next, now, a.scale_log2, p);
            core.template add_values<false>(v_tile(t), p, odd);
            if (t + 2 == n_c) mask(next, up_to(Lc - (t + 1) * CORE_KEYS));
        };
        f32x16 next[2];
        for (; t + 2 < c_end; t += 2) {                                         // (two at a time: scores stay where they are)
            turn(t, s, next);
            turn(t + 1, next, s);
        }
        if (t + 1 < c_end) {
            turn(t++, s, next);
            s[0] = next[0];
            s[1] = next[1];
        }
        meet();
        if (!idle) {
            core.probabilities(s, a.scale_log2, p, false);
            core.template add_values<false>(v_tile(t), p, odd);
        }
        t++;
    }
    // ---- the prefix and the pass' rows: bf16, not seen by every query
    const int t_odd = t;
    auto rows_of = [&](int t, const uint16_t *&k, const uint16_t *&v, int64_t &ldk, int64_t &ldv, int &n, uint64_t &sees) __attribute__((always_inline)) {
        const bool in_prefix = t < n_c + n_p;
        const int key0 = CORE_KEYS * (in_prefix ? t - n_c : t - n_c - n_p);
        ldk = in_prefix ? HD : a.k_at.row;
        ldv = in_prefix ? HD : a.v_at.row;
        k = in_prefix ? a.prompt_k + (int64_t)h * a.P * HD : a.k_rows + a.k_at.at(b, h, 0);
        v = in_prefix ? a.prompt_v + (int64_t)h * a.P * HD : a.v_rows + a.v_at.at(b, h, 0);
        k += key0 * ldk;
        v += key0 * ldv;
        n = (in_prefix ? a.P : a.R) - key0;
        const int row = query_now() / a.qpk;
        sees = (in_prefix ? (a.t.is_mask[row] ? ~0ull : 0) : a.t.anc[(int64_t)row * a.t.words + (key0 >> 6)]) & up_to(n);
    };
    for (; t < end; t++) {
        const uint16_t *k, *v;
        int64_t ldk, ldv;
        int n;
        uint64_t sees;
        rows_of(t, k, v, ldk, ldv, n, sees);
        const int l = core_lane(), r = min(16 * wave + (l & 15), n - 1), first = VPL * (l >> 4);
        bf16x8 x[PARTS], y[PARTS];
#pragma unroll
        for (int i = 0; i < PARTS; i++) {
            x[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(k + r * ldk + first + 8 * i));
            y[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(v + r * ldv + first + 8 * i));
        }
        meet();
        put(k_tile(t), false, x);
        put(v_tile(t), true, y);
        meet();
        if (idle) continue;
        core.scores(k_tile(t), s);
        mask(s, sees);
        core.probabilities(s, a.scale_log2, p, true);
        core.template add_values<true>(v_tile(t), p, odd);
    }
    if (__builtin_amdgcn_ballot_w64(odd != 0) != 0)
        for (t = t_odd; t < end; t++) {
            const uint16_t *k, *v;
            int64_t ldk, ldv;
            int n;
            uint64_t sees;
            rows_of(t, k, v, ldk, ldv, n, sees);
            core.add_nonfinite(v, ldv, n - 1, sees);
        }

    const int end_lane = core_lane(), qi = tile * AMW_ROWS + wave * 32 + (end_lane & 31), half = end_lane >> 5;
    if (qi >= nq) return;
    const AmxArgs z = amx_again();
    const int row = qi / z.qpk, head = h * z.qpk + (qi - row * z.qpk);
    const float l = core_sum_halves(core.l_run);
    const bool absent = z.token && !z.t.is_mask[row] && z.token[(int64_t)b * z.R + row] < 0;
    if (at.split) {                                                             // unnormalised: for attn_mx_merge_kernel
        // The sum's own power of two goes to the exponent: shares are weighed by what they hold, whatever reference they used (0 for what is no number).
        const int e = __builtin_amdgcn_frexp_expf(l);
        const int64_t to = z.part(at.share, row, head);
        float *dst = z.part_o + to * HD + 4 * half;
#pragma unroll
        for (int n = 0; n < Core::NT; n++)
#pragma unroll
            for (int i = 0; i < 4; i++)
                *reinterpret_cast<float4 *>(dst + 32 * n + 8 * i) =
                    make_float4(ldexpf(core.o[n][4 * i], -e), ldexpf(core.o[n][4 * i + 1], -e), ldexpf(core.o[n][4 * i + 2], -e), ldexpf(core.o[n][4 * i + 3], -e));
        if (half == 0) *reinterpret_cast<float2 *>(z.part_ml + to * 2) = absent || l == 0.f ? make_float2(-INFINITY, 0.f) : make_float2(core.base + e, ldexpf(l, -e));
        return;
    }
    // (an absent row gives zeros, and a sum of nothing)
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    uint16_t *dst = z.out + z.query(b, row, head) * HD;
    core.put(dst, inv, half);
    if (absent) {
#pragma unroll
        for (int i = 0; i < HD / 16; i++) *reinterpret_cast<uint4 *>(dst + 8 * (2 * i + half)) = make_uint4(0, 0, 0, 0);
    }
}

// o = sum_s w_s o_s / sum_s w_s l_s, w_s = 2^(m_s - max m): HD / 4 threads a query's columns, SIDE such rows of threads side by side its shares (and
// in a workgroup of 256 or more threads as many queries as there is room for).  A share without keys for the query has m = -inf and is left out
// (nothing of it need have been written).  Bound by what the shares left in memory: 12 shares of 4352 queries 6.3 us, 27 MB; few of them: by a launch and two ways to memory, 4.1.
template <int HD, int SIDE, int THREADS>
__global__ __launch_bounds__(THREADS) void attn_mx_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml, const int2 *__restrict__ share_of, int64_t n_queries,
                                                                int of_sequence, int stride, int n_shares, uint16_t *__restrict__ out) {
    constexpr int LANES = HD / 4, QUERIES = THREADS / (LANES * SIDE);
    const int i = threadIdx.x % LANES, side = threadIdx.x / LANES % SIDE, mine = threadIdx.x / (LANES * SIDE);
    const int64_t qrow = (int64_t)blockIdx.x * QUERIES + mine;
    const bool ok = qrow < n_queries;
    const int b = (uint32_t)(ok ? qrow : 0) / (uint32_t)of_sequence;            // (there are fewer than 2^27 queries)
    const int2 shares = share_of[b];
    const int n_splits = n_shares ? n_shares : shares.y;                        // (one sequence: its parts are on their way before it is known how many there are)
    const int64_t part = (int64_t)(n_shares ? 0 : shares.x) * of_sequence + ((ok ? qrow : 0) - (int64_t)b * of_sequence), step = (int64_t)stride * of_sequence;
    const float2 *ml = reinterpret_cast<const float2 *>(part_ml) + part;
    const float4 *po = reinterpret_cast<const float4 *>(part_o + part * HD) + i;
    float m = -INFINITY, l = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = side; s0 < n_splits; s0 += 4 * SIDE) {                        // four shares of a thread at a time, against their own maximum
        float2 e[4];
        float4 o[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int s = min(s0 + k * SIDE, n_splits - 1);
            e[k] = ml[s * step];
            o[k] = po[s * step * LANES];
            if (s0 + k * SIDE >= shares.y) e[k].x = -INFINITY;
        }
        const float m_new = fmaxf(fmaxf(fmaxf(e[0].x, e[1].x), fmaxf(e[2].x, e[3].x)), m);
        if (m_new == -INFINITY) continue;
        const float f = amx_exp2(m - m_new);
        l *= f;
        x.x *= f; x.y *= f; x.z *= f; x.w *= f;
        m = m_new;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            if (e[k].x == -INFINITY) continue;
            const float w = amx_exp2(e[k].x - m);
            l += w * e[k].y;
            x.x += w * o[k].x; x.y += w * o[k].y; x.z += w * o[k].z; x.w += w * o[k].w;
        }
    }
    if constexpr (SIDE > 1) {
        __shared__ float4 s_o[QUERIES][SIDE][LANES];
        __shared__ float2 s_ml[QUERIES][SIDE];
        s_o[mine][side][i] = x;
        if (i == 0) s_ml[mine][side] = make_float2(m, l);
        __syncthreads();
        if (side) return;
        float top = m;
        for (int k = 1; k < SIDE; k++) top = fmaxf(top, s_ml[mine][k].x);
        l = 0.f;
        x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int k = 0; k < SIDE; k++) {
            const float2 e = s_ml[mine][k];
            if (e.x == -INFINITY) continue;
            const float w = amx_exp2(e.x - top);
            const float4 y = s_o[mine][k][i];
            l += w * e.y;
            x.x += w * y.x; x.y += w * y.y; x.z += w * y.z; x.w += w * y.w;
        }
        m = top;
    }
    if (!ok || shares.y == 1) return;                                           // (one share: it wrote the result itself)
    const float inv = 1.0f / l;
    *reinterpret_cast<uint2 *>(out + qrow * HD + 4 * i) =
        m == -INFINITY ? make_uint2(0, 0) : make_uint2(amx_pk_bf16(x.x * inv, x.y * inv), amx_pk_bf16(x.z * inv, x.w * inv));
}
template <int HD>
static void launch_merge(const AmxArgs &a, int64_t queries, hipStream_t s) {
    const int of_sequence = a.R * a.qpk * a.kv.Hkv, stride = a.kv.batch > 64 ? a.kv.batch : 1, n = (a.n_shares + a.kv.batch - 1) / a.kv.batch, one = a.kv.batch == 1 ? a.n_shares : 0;
    // few shares: a thread takes them all; many: 8 or 32 rows of threads share them
    if (n <= 8) hipLaunchKernelGGL((attn_mx_merge_kernel<HD, 1, 256>), dim3((unsigned)((queries * HD / 4 + 255) / 256)), dim3(256), 0, s, a.part_o, a.part_ml, a.share_of, queries, of_sequence, stride, one, a.out);
    else if (n <= 32) hipLaunchKernelGGL((attn_mx_merge_kernel<HD, 8, 256>), dim3((unsigned)((queries * HD / 4 * 8 + 255) / 256)), dim3(256), 0, s, a.part_o, a.part_ml, a.share_of, queries, of_sequence, stride, one, a.out);
    else hipLaunchKernelGGL((attn_mx_merge_kernel<HD, 32, HD * 8>), dim3((unsigned)queries), dim3(HD * 8), 0, s, a.part_o, a.part_ml, a.share_of, queries, of_sequence, stride, one, a.out);
}

struct AmxPlan { bool wide; int tiles_u, waves, n_tiles, shares, per_share; int64_t workgroups; size_t part_o, part_ml, total; };

// How a launch is cut, from nothing but its sizes: 16 queries a workgroup of 8 waves or of 4, 32 queries, or 128 that share decoded keys (wide); and how many shares the
// keys of all sequences are split into (as many as sequences: not at all).  The estimate behind the choice, in us at head_dim 128:
//   a round of workgroups: their start and end, and their turns (256 keys, 128, 128, 64) at the pace of one workgroup a CU or of as many as a CU holds, but no faster
//   than a CU takes codes in, 35 KB a us; the bytes that all of them read at 6 TB/s, 5 where tiles of queries read the same ones again (of these two the longer, and a
//   quarter of the other); and, where the keys are split, a second kernel and what the shares write and read, at 9 TB/s (it is still in a cache: 12 shares of 4352 queries 6 us).
// Split launches fill the card once (three workgroups of 16 queries and 4 waves a CU; of 8 bits at head_dim 128 a CU holds two, but shares cut for two were no better).
// A batch's lengths are taken to be half to three quarters of the hint on average; not split, its longest decides.  Where sequences are alike instead, amx_place, whose
// shares have one size, gives each as many as fit for all and leaves the rest empty (17 sequences and 32 shares: one each); what that costs more counts for three tenths.
// Without that, equal lengths: 17 sequences of 8192 keys, 64/8 heads, 46 us at 4 bits and 78 at 8 (now 35 and 59), 33 at 8 bits 164 (138), four trees of 68 rows over 3000 keys 80
// (51), of 5 sequences of 4096, 32/32 heads, 8 bits 43 (36); what it took where lengths differ: 33 sequences of 8 bits 66 (77), 8 of 4096, 32/32 heads 23 (26), most others nothing.
// Measured (16 queries in 4 waves / 32 / wide): a turn with one workgroup a CU 0.9 / 1.25 / 1.37 us, with two 1.44 / 2.1 / 2.1; the start and end 5.6 / 5.6 / 7; a turn of
// 8 waves 1.0.  Each kind with its best shares, 16 queries in 8 waves / in 4 / 32 / wide:
//   68 rows, 32 heads of their own keys, 1024 keys of 4 bits 11.9 / 14.3 / 15.9 / 19.4 us; 4096 keys of 8 bits 42 / 40 / 30 / 25; four sequences of 400 to 1100
//   keys 31.7 / 21.5 / 29.1 / 29.3; 4 sequences of 1024 to 4096 keys, 64/8 heads 146 / 127 / 82 / 54; 20 rows there 39 / 32 / 30 / 32; single tokens: 32 sequences
//   of up to 8192 keys 42 / 32.5 / 44 / 67; one of 131072 keys of 4 bits 31 / 37 / 42 / 62; one of 1000, 32 heads 9.8 / 10.0 / 10.6 / 12 (the last three with
//   a second kernel, whose launch costs the host as much again: hence 3.5 us for it, more than its own time).
// With shares cut from the hint instead, 8 sequences of 100 to 4000 keys of 8 bits, 32 heads, took 43 us (now 29), 3 of 0 to 39168, 6/2 heads 28 (17), 30 of 0 to
// 26000 45 (37), the 32 above 36.
static AmxPlan amx_plan(int batch, int rows, int Hq, int Hkv, int hd, int bits, int ctx_hint, int n_prompt) {
    static const struct { int queries, unit, waves, slots; double start, one, many; } kinds[4] = {
        {16, AMX_CHUNK, 8, 256, 5.6, 1.0, 1.0}, {16, AMX_CHUNK, 4, 768, 5.6, 0.9, 1.44}, {32, AMX_CHUNK, 4, 512, 5.6, 1.25, 2.1}, {AMW_ROWS, CORE_KEYS, 4, 512, 7.0, 1.37, 2.1}};
    static const int per_sequence[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 80, 96, 128, 192, 256};
    const int64_t nq = (int64_t)rows * (Hq / Hkv);
    const double size = hd / 128.0, key_bytes = 2 * (hd * bits / 8 + hd / 32), keys = (double)batch * Hkv * ctx_hint * key_bytes;
    AmxPlan p = {};
    double best = 1e300;
    for (int k = 0; k < (nq <= 16 ? 2 : nq <= 32 ? 3 : 4); k++) {
        const auto &kind = kinds[k];
        const int unroll = k == 3 ? 1 : kind.waves;                             // chunks of a turn
        const int n_tiles = (int)((nq + kind.queries - 1) / kind.queries);
        auto units = [&](int64_t n) { return (n + kind.unit - 1) / kind.unit; };
        auto turns_of = [&](int64_t n) { return (units(n_prompt) + units(n) + units(rows) + unroll - 1) / unroll; };
        const int64_t longest = turns_of(ctx_hint), usual = turns_of(batch > 1 ? (int64_t)(0.6 * ctx_hint) : ctx_hint), share_wgs = (int64_t)Hkv * n_tiles;
        // of sequences that are alike, all as long as the hint, or of lengths that differ
        auto estimate = [&](int64_t shares, int64_t per, bool alike) {
            const bool split = shares > batch;
            double turns = (double)longest, wgs = (double)shares * share_wgs;
            if (split && batch > 64) turns = (double)per;
            else if (split && alike) {                                          // every sequence has as many shares, and the rest has nothing to do
                const int64_t p = (longest + shares / batch - 1) / (shares / batch);
                turns = (double)p;
                wgs = (double)((longest + p - 1) / p * batch * share_wgs);
            } else if (split) turns = (double)(usual * batch + shares - 1) / shares + (batch > 1 ? 0.5 : 0.0);
            // (not split, a batch's short sequences leave room for others; alone on a CU, a workgroup leaves it to the next one late)
            const double busy = wgs * (k && batch > 1 && !alike && (!split || batch > 64) ? 0.75 : 1.0);
            const double rounds = k && batch > 1 ? std::max(busy / kind.slots, 1.0) : std::ceil(wgs / kind.slots);
            const double on_a_cu = std::min(std::max(split && batch <= 64 ? std::ceil(busy / 256) : busy / 256, 1.0), kind.slots / 256.0);
            const double turn = std::max(size * (busy <= 256 ? kind.one : kind.many), on_a_cu * unroll * kind.unit * key_bytes / 35e3);
            const double pace = rounds * turns * turn, load = keys * (batch > 1 && !alike ? 0.5 : 1.0) * n_tiles / (n_tiles > 1 ? 5e6 : 6e6);
            double us = rounds * kind.start + std::max(pace, load) + 0.25 * std::min(pace, load);
            if (split) us += 3.5 + 0.03 * (double)shares / batch + (double)shares * rows * Hq * hd * 8 / 9e6;
            return us;
        };
        auto consider = [&](int64_t shares, int64_t per) {
            double us = estimate(shares, per, false);
            if (batch > 1 && batch <= 64) us += 0.3 * std::max(estimate(shares, per, true) - us, 0.0);
            if (us < best) {
                best = us;
                p.wide = k == 3;
                p.tiles_u = k < 2 ? 1 : 2;
                p.waves = kind.waves;
                p.n_tiles = n_tiles;
                p.shares = (int)shares;
                p.per_share = (int)per;
                p.workgroups = shares * share_wgs;
            }
        };
        for (int want : per_sequence) {
            const int64_t per = (longest + want - 1) / want, shares = (longest + per - 1) / per * batch;
            if (want > 1 && (want > longest || shares * share_wgs > kind.slots * (batch > 64 ? 2 : 1))) break;
            consider(shares, per);
        }
        if (batch <= 64)                                                        // as many as a CU, or two of them, or three hold
            for (int slots = 256; slots <= kind.slots; slots += 256)
                if (slots / share_wgs > batch && slots / share_wgs <= batch * longest) consider(slots / share_wgs, 0);
    }
    if (p.shares > batch) {
        auto up = [](size_t n) { return (n + 255) / 256 * 256; };
        p.part_o = up((size_t)p.shares * rows * Hq * hd * 4);
        p.part_ml = up((size_t)p.shares * rows * Hq * 8);
        p.total = p.part_o + p.part_ml + up((size_t)batch * 8);
    }
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
    const AmxPlan p = amx_plan(batch, rows, n_heads, n_kv_heads, head_dim, bits, ctx_hint, n_prompt);
    return p.total;
}

extern "C" int bita_tree_attention_mx_plan_info(int32_t batch, int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t bits, int32_t ctx_hint,
                                                int32_t n_prompt, int32_t *out4) {
    if (!out4) return bita_set_error(BITA_ERR_INVALID_ARG, "bita_tree_attention_mx_plan_info: null argument");
    if (int rc = amx_sizes("bita_tree_attention_mx_plan_info", batch, rows, n_heads, n_kv_heads, head_dim, bits, ctx_hint, n_prompt)) return rc;
    const AmxPlan p = amx_plan(batch, rows, n_heads, n_kv_heads, head_dim, bits, ctx_hint, n_prompt);
    out4[0] = (p.shares + batch - 1) / batch; out4[1] = p.wide ? AMW_ROWS : 16 * p.tiles_u; out4[2] = p.waves;
    out4[3] = p.workgroups < INT32_MAX ? (int32_t)p.workgroups : INT32_MAX;
    return BITA_OK;
}

template <int HD, int BITS>
static void launch_amw(const AmxArgs &a, int64_t n_units, hipStream_t s) {
    const dim3 grid((unsigned)((n_units + 7) / 8 * 8 * a.n_tiles));
    hipLaunchKernelGGL((attn_mx_wide_kernel<HD, BITS>), grid, dim3(AMX_WAVES * 64), (4 * AttnCore<HD>::TILE), s, a);
}
template <int HD, int BITS, int U, int W>
static void launch_amx(const AmxArgs &a, int64_t n_units, hipStream_t s) {
    constexpr int SMEM = AmxCfg<HD, U, W>::SMEM;
    static_assert(W / AMX_WAVES * SMEM <= 160 * 1024 && SMEM <= 80 * 1024, "two workgroups a CU");
    if (SMEM > 64 * 1024) (void)hipFuncSetAttribute((const void *)attn_mx_kernel<HD, BITS, U, W>, hipFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    const dim3 grid((unsigned)((n_units + 7) / 8 * 8 * a.n_tiles));
    hipLaunchKernelGGL((attn_mx_kernel<HD, BITS, U, W>), grid, dim3(W * 64), SMEM, s, a);
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
    a.k_at = mx_rows(kv->batch, k_seq, kv->n_kv_heads, k_head, t->dev.rows, k_row);
    a.v_at = mx_rows(kv->batch, v_seq, kv->n_kv_heads, v_head, t->dev.rows, v_row);
    if (int rc = mx_rows_check(who, a.k_at, a.v_at, (uintptr_t)d_q | (uintptr_t)d_k_rows | (uintptr_t)d_v_rows | (uintptr_t)d_prompt_k | (uintptr_t)d_prompt_v |
                                                        (uintptr_t)d_out | (uintptr_t)d_ws)) return rc;
    const AmxPlan p = amx_plan(kv->batch, t->dev.rows, n_heads, kv->n_kv_heads, kv->head_dim, kv->bits, ctx_hint, n_prompt);
    if (ws_bytes < p.total || (p.total && !d_ws)) return bita_set_error(BITA_ERR_CAPACITY, "%s: workspace %zu < %zu bytes", who, ws_bytes, p.total);
    a.t = t->dev;
    a.q = (const uint16_t *)d_q; a.k_rows = (const uint16_t *)d_k_rows; a.v_rows = (const uint16_t *)d_v_rows;
    a.prompt_k = (const uint16_t *)d_prompt_k; a.prompt_v = (const uint16_t *)d_prompt_v;
    a.ctx_len = d_ctx_len; a.token = d_token;
    a.P = n_prompt; a.R = t->dev.rows; a.qpk = n_heads / kv->n_kv_heads; a.ctx_hint = ctx_hint;
    a.n_tiles = p.n_tiles; a.n_shares = p.shares; a.per_share = p.per_share;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)kv->head_dim);
    a.part_o = (float *)d_ws; a.part_ml = (float *)((unsigned char *)d_ws + p.part_o);
    a.share_of = (int2 *)((unsigned char *)d_ws + p.part_o + p.part_ml);
    a.out = (uint16_t *)d_out;
    hipStream_t s = (hipStream_t)stream;
    const int64_t units = (int64_t)p.shares * kv->n_kv_heads;
#define AMX_LAUNCH(HD_, BITS_) do { if (p.wide) launch_amw<HD_, BITS_>(a, units, s); else if (p.tiles_u == 2) launch_amx<HD_, BITS_, 2, 4>(a, units, s); \
    else if (p.waves == 8) launch_amx<HD_, BITS_, 1, 8>(a, units, s); else launch_amx<HD_, BITS_, 1, 4>(a, units, s); } while (0)
    if (kv->head_dim == 128) { if (kv->bits == 4) AMX_LAUNCH(128, 4); else AMX_LAUNCH(128, 8); }
    else { if (kv->bits == 4) AMX_LAUNCH(64, 4); else AMX_LAUNCH(64, 8); }
#undef AMX_LAUNCH
    if (p.shares > kv->batch) {
        const int64_t queries = (int64_t)kv->batch * t->dev.rows * n_heads;
        if (kv->head_dim == 128) launch_merge<128>(a, queries, s);
        else launch_merge<64>(a, queries, s);
    }
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}
