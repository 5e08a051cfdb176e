// Causal attention over packed prompts: o_i = sum_{j <= i} softmax_j(q_i k_j / sqrt(d)) v_j inside every sequence.
//
// A workgroup owns 128 queries of one head, 32 a wave, and walks the keys in tiles of 64 up to its last query, with a running maximum
// and sum per query.
//  * S^T = K Q^T by 32 x 32 x 16 matrix instructions: a lane has 32 of its query's 64 scores, the other half wave the rest, so a maximum or a sum
//    crosses lanes once.  The layout of S^T is the B operand of O^T = V^T P^T when that takes the keys in the order in which S^T
//    holds them (lane half h: keys 8 i + 4 h + 0..3): the probabilities stay in registers.
//  * K and V tiles go from memory to LDS without passing registers, into one of two buffers, while the other is multiplied (K two tiles ahead of
//    the values, V one: scores run a tile ahead); one barrier a tile.  Rows are swizzled by 16-byte columns on the way (by where a lane fetches from: LDS takes them in lane order),
//    K is read back by rows, V by transposed reads.
//  * Key tiles before a wave's queries need no mask.  Workgroups start with the longest walks.
// Bound by matrix instructions at the clock that the card holds under them, with the exponentials between them: 8192 tokens of 64/8 heads of 128 1015 us, 1083 TFLOP/s
// of what the mask leaves, 0.91 of the library's rate for a product of 8192^3 (964 on another card); a turn of two workgroups on a CU 1.95 us.  Ragged prompts by the packing of their walks: 2049, 1411, 977,
// 350 tokens and less of 32 heads 80 us, 74 of them a packing without starts and ends.
#include <cmath>
#include <type_traits>
#include "attention_core.h"

#define PA_WAVES 4
#define PA_ROWS (32 * PA_WAVES)
#define PA_SKIP 8
#define PA_MAX_LD (1 << 24)            // offsets inside a tile of 64 rows have 32 bits (signed)

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t ldq, q_head, ldk, k_head, ldv, v_head, ldo;
    const int32_t *cu;
    int n_seqs, n_tokens, Hq, qpk;
    float scale_log2;
    uint16_t *out;
};

// f over all lanes (a sum, a maximum; 0 is its neutral element): rows of 16 lanes by rotation, then the four rows
template <typename F>
__device__ __forceinline__ int pa_over_wave(int x, F &&f) {
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x121, 0xF, 0xF, false));        // row_ror 1, 2, 4, 8
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x122, 0xF, 0xF, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x124, 0xF, 0xF, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, false));
    return f(f(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16)), f(__builtin_amdgcn_readlane(x, 32), __builtin_amdgcn_readlane(x, 48)));
}

// The workgroup's tile of queries: its sequence's first token and length, and its number in the sequence.  Tiles count from the longest walk
// down, over 64 sequences (a lane each) at a time: of every number the tiles that sequences have, until `tile` is reached.  false: no such tile.
__device__ __forceinline__ bool pa_find(const PromptArgs &a, int tile, int &start, int &len, int &mine) {
    const int lane = threadIdx.x & 63;
    auto sequence = [&](int b, int &s, int &n) __attribute__((always_inline)) {
        s = n = 0;
        if (b < a.n_seqs) {
            s = min(max(a.cu[b], 0), a.n_tokens);
            n = min(max(a.cu[b + 1], s), a.n_tokens) - s;
        }
        return (n + PA_ROWS - 1) / PA_ROWS;
    };
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        while (a.n_seqs - b0 > PA_SKIP * 64) {                                          // (of very many, 8 a lane are passed over at a time)
            int s, n, all = 0;
#pragma unroll
            for (int i = 0; i < PA_SKIP; i++) all += sequence(b0 + 64 * i + lane, s, n);
            all = pa_over_wave(all, [](int x, int y) { return x + y; });
            if (tile < all) break;
            tile -= all;
            b0 += PA_SKIP * 64;
        }
        int s, n;
        const int tiles = sequence(b0 + lane, s, n);
        const int all = pa_over_wave(tiles, [](int x, int y) { return x + y; }), most = pa_over_wave(tiles, [](int x, int y) { return max(x, y); });
        if (tile >= all) {
            tile -= all;
            continue;
        }
        for (int k = most - 1;; k--) {                                                 // (ends: `all` is the sum of these counts over k)
            const uint64_t has = __builtin_amdgcn_ballot_w64(tiles > k);
            const int count = __popcll(has);
            if (tile >= count) {
                tile -= count;
                continue;
            }
            // the lane that has `tile` others before it
            const bool me = tiles > k && __popcll(has & ((1ull << lane) - 1)) == tile;
            const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(me));
            start = __builtin_amdgcn_readlane(s, at);
            len = __builtin_amdgcn_readlane(n, at);
            mine = k;
            return true;
        }
    }
    return false;
}

// (of narrow heads a CU holds three workgroups: 8192 tokens of 64/8 heads of 64 in 590 us, with two 616, when both were timed, now 583; nine packed prompts of 32 heads 51, with two 54.7, now 46.5)
template <int HD>
__global__ __launch_bounds__(PA_WAVES * 64, HD == 64 ? 3 : 2) void prompt_attn_kernel(PromptArgs a) {
    using Core = AttnCore<HD>;
    constexpr int KS = Core::KS, TILE = Core::TILE, GPR = HD / 8, RPI = 64 / GPR;    // granules a row, rows a load instruction
    constexpr int LOADS = CORE_KEYS / RPI / PA_WAVES;                                   // load instructions of a wave, K or V tile
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];              // K tiles [2], V tiles [2]
    const int lane = threadIdx.x & 63, hf = lane >> 5, c = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j = blockIdx.x % a.Hq;
    const int head = a.Hq % 8 == 0 ? (j & 7) * (a.Hq >> 3) + (j >> 3) : j;              // an XCD (ids go round) takes neighbouring heads
    int start, len, tile;
    if (!pa_find(a, blockIdx.x / a.Hq, start, len, tile)) return;                       // (the same in all lanes, and the compiler knows)
    const int q0 = tile * PA_ROWS + wave * 32, qi = q0 + c, kvh = head / a.qpk;         // of the wave, of the lane: inside the sequence
    const int64_t qrow = start + min(qi, len - 1);

    Core core;
    core.init(lane);
#pragma unroll
    for (int s = 0; s < KS; s++)
        core.q[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(a.q + qrow * a.ldq + head * a.q_head + 16 * s + 8 * hf));

    const int n_tiles = (min(len, (tile + 1) * PA_ROWS) + CORE_KEYS - 1) / CORE_KEYS;
    const int n_whole = q0 / CORE_KEYS;                                                 // tiles that all of the wave's queries see whole
    const uint16_t *kbase = a.k + (int64_t)start * a.ldk + kvh * a.k_head, *vbase = a.v + (int64_t)start * a.ldv + kvh * a.v_head;
    const uint32_t lds = (uint32_t)(size_t)((__attribute__((address_space(3))) unsigned char *)smem);
    // The wave's part of a tile is rows wave * 64 / PA_WAVES .., RPI of them an instruction: a descriptor at the tile's first row (what lies behind the
    // sequence's last one is out of its range, and 0), the instruction's row in the scalar offset, this lane's row and column in two
    // registers; the swizzle's share of the instruction's row is an exclusive or.
    constexpr int R0 = CORE_KEYS / PA_WAVES, K_STEP = 4, V_STEP = HD == 128 ? 1 : 2;
    const int lr = lane / GPR, lp = lane % GPR;
    const uint32_t k_row = lr * (uint32_t)a.ldk * 2, k_col = (lp ^ Core::k_swizzle(lr)) * 16;
    const uint32_t v_row = lr * (uint32_t)a.ldv * 2, v_col = (lp ^ Core::v_swizzle(lr)) * 16;
    auto fetch = [&](int t, bool is_v) __attribute__((always_inline)) {
        unsigned char *dst = smem + (is_v ? 2 * TILE : 0) + (t & 1) * TILE + wave * (TILE / PA_WAVES);
        const uint32_t ld = 2 * (uint32_t)(is_v ? a.ldv : a.ldk), rows = min(len - t * CORE_KEYS, CORE_KEYS);
        const __amdgpu_buffer_rsrc_t rsrc =
            __builtin_amdgcn_make_buffer_rsrc((void *)((is_v ? vbase : kbase) + (int64_t)t * CORE_KEYS * (is_v ? a.ldv : a.ldk)), 0, (rows - 1) * ld + HD * 2, 0x00027000);
#pragma unroll
        for (int i = 0; i < LOADS; i++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(dst + i * 1024), 16,
                                                     is_v ? (v_col ^ (16 * V_STEP * i)) + v_row : (k_col ^ (16 * K_STEP * i)) + k_row, (R0 * wave + RPI * i) * ld, 0, 0);
    };
    auto landed = [&](auto behind) __attribute__((always_inline)) {                     // everyone's loads but the last few are in LDS, everyone's reads are done
        __builtin_amdgcn_s_waitcnt(0x0070 + decltype(behind)::value);                   // vmcnt(behind), lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto k_tile = [&](int t) __attribute__((always_inline)) { return lds + (t & 1) * TILE; };
    auto v_tile = [&](int t) __attribute__((always_inline)) { return lds + 2 * TILE + (t & 1) * TILE; };
    auto mask = [&](int t, f32x16 (&s)[2]) __attribute__((always_inline)) {
        int last = qi - t * CORE_KEYS - 4 * hf;                                         // of the keys 8 i + r that this lane holds
        asm volatile("" : "+v"(last));
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int e = 0; e < 16; e++) s[h][e] = 32 * h + 8 * (e >> 2) + (e & 3) <= last ? s[h][e] : -INFINITY;
    };

    auto turn = [&](int t) __attribute__((always_inline)) {                             // tile t's V and t + 1's K are there; the next are asked for
        landed(std::integral_constant<int, 0>{});
        if (t + 2 < n_tiles) fetch(t + 2, false);
        if (t + 1 < n_tiles) fetch(t + 1, true);
    };

    // Scores run a tile ahead: while a tile's become probabilities, the matrix cores work on the next one's.  So K is fetched two tiles
    // ahead, V one.  A wave's queries lie in one tile of keys: those before it are seen whole, behind it there is only the others' pace to keep.
    f32x16 s[2];
    uint32_t p[16], odd = 0;
    int t = 0;
    static_assert(2 * LOADS < 16, "the count of a wait");
    asm volatile("" ::: "memory");                                                      // (the queries are asked for before the tiles: the wait below counts what is behind K's first)
    __builtin_amdgcn_sched_barrier(0);
    fetch(0, false);
    fetch(0, true);
    if (n_tiles > 1) {
        fetch(1, false);
        landed(std::integral_constant<int, 2 * LOADS>{});
    } else landed(std::integral_constant<int, LOADS>{});
    if (q0 < len) {
        core.scores(k_tile(0), s);
        if (n_whole == 0) mask(0, s);
        core.take_maximum(core.largest(s), a.scale_log2);                               // (what every query's reference starts with)
        auto whole = [&](int t, f32x16 (&now)[2], f32x16 (&next)[2]) __attribute__((always_inline)) {
            turn(t);
            core.scores_and_probabilities(k_tile(t + 1), next, now, a.scale_log2, p);
            core.template add_values<false>(v_tile(t), p, odd);
        };
        f32x16 next[2];
        for (; t + 2 <= n_whole; t += 2) {                                              // (two at a time: scores stay where they are)
            whole(t, s, next);
            whole(t + 1, next, s);
        }
        if (t < n_whole) {
            whole(t++, s, next);
            s[0] = next[0];
            s[1] = next[1];
        }
        turn(t);
        mask(t, s);
        core.probabilities(s, a.scale_log2, p, false);
        core.template add_values<true>(v_tile(t), p, odd);
        if (__builtin_amdgcn_ballot_w64(odd != 0) != 0) {
            const int past = qi - t * CORE_KEYS;                                        // keys 0 .. past of the tile are seen
            core.add_nonfinite(vbase + (int64_t)t * CORE_KEYS * a.ldv, a.ldv, len - 1 - t * CORE_KEYS, past >= 63 ? ~0ull : (2ull << past) - 1);
        }
        t++;
    }
    for (; t < n_tiles; t++) turn(t);
    const float inv = 1.0f / core_sum_halves(core.l_run);
    const int end_lane = core_lane(), query = q0 + (end_lane & 31);
    if (query < len) core.put(a.out + (int64_t)(start + query) * a.ldo + (int64_t)head * HD, inv, end_lane >> 5);
}

extern "C" int bita_prompt_attention(const void *d_q, int64_t ldq, int64_t q_head_stride, const void *d_k, int64_t ldk, int64_t k_head_stride,
                                     const void *d_v, int64_t ldv, int64_t v_head_stride, const int32_t *d_cu_seqlens, int32_t n_seqs, int32_t n_tokens,
                                     int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, void *d_out, int64_t ldo, void *stream) {
    const char *who = "bita_prompt_attention";
    if ((n_tokens && (!d_q || !d_k || !d_v || !d_out)) || !d_cu_seqlens || n_seqs <= 0 || n_tokens < 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads)
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: null argument, non-positive or inconsistent size", who);
    if (head_dim != 64 && head_dim != 128) return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128", who);
    if (n_tokens <= 1) ldq = ldk = ldv = 0, ldo = (int64_t)n_heads * head_dim;                  // (strides of axes with one place are nobody's)
    if (n_heads == 1) q_head_stride = 0;
    if (n_kv_heads == 1) k_head_stride = v_head_stride = 0;
    if (ldq < 0 || ldk < 0 || ldv < 0 || q_head_stride < 0 || k_head_stride < 0 || v_head_stride < 0 || ldo < (int64_t)n_heads * head_dim)
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: negative stride, or output rows of %lld values %lld apart", who, (long long)n_heads * head_dim, (long long)ldo);
    if ((ldq | ldk | ldv | q_head_stride | k_head_stride | v_head_stride | ldo) & 7 ||
        ((uintptr_t)d_q | (uintptr_t)d_k | (uintptr_t)d_v | (uintptr_t)d_out) & 15)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: strides must be multiples of 8 elements, pointers of 16 bytes", who);
    if (ldk > PA_MAX_LD || ldv > PA_MAX_LD) return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: rows of k and v at most %d elements apart", who, PA_MAX_LD);
    const int64_t tiles = (int64_t)n_tokens / PA_ROWS + n_seqs, wgs = tiles * n_heads;          // no tiling of the sequences has more
    if (wgs > (int64_t)((1ull << 32) / (PA_WAVES * 64)) - 1)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: %lld workgroups", who, (long long)wgs);
    if (n_tokens == 0) return BITA_OK;
    const PromptArgs a = {(const uint16_t *)d_q, (const uint16_t *)d_k, (const uint16_t *)d_v, ldq, q_head_stride, ldk, k_head_stride, ldv, v_head_stride, ldo,
                          d_cu_seqlens, n_seqs, n_tokens, n_heads, n_heads / n_kv_heads, 1.4426950408889634f / sqrtf((float)head_dim), (uint16_t *)d_out};
    hipStream_t s = (hipStream_t)stream;
    if (head_dim == 128) hipLaunchKernelGGL((prompt_attn_kernel<128>), dim3((unsigned)wgs), dim3(PA_WAVES * 64), 4 * AttnCore<128>::TILE, s, a);
    else hipLaunchKernelGGL((prompt_attn_kernel<64>), dim3((unsigned)wgs), dim3(PA_WAVES * 64), 4 * AttnCore<64>::TILE, s, a);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}
