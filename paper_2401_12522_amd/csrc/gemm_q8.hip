// The product of 8-bit integers with scales: Y[m][n] = (sum_k A[m][k] W[n][k]) sa[m] sw[n], sums in 32-bit integers.
#include "common.h"
#include <atomic>
#include <cmath>

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

// (stores of 8 and 16 bytes at an element's alignment: the hardware takes them)
struct __attribute__((packed, aligned(4))) Words4 { float v[4]; };
struct __attribute__((packed, aligned(2))) Halves4 { uint16_t v[4]; };

// Four neighbouring columns of one row: sums times scales.  The product of the sum and the row's scale is rounded to fp32, then
// its product with the column's, as a row factor and a column factor would be applied one after the other.
__device__ __forceinline__ void store4(void *out, int out_type, int64_t ldo, int row, int64_t col, int64_t n, i32x4 acc, float sa, const float *__restrict__ sw) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = (float)acc[e] * sa * (col + e < n ? sw[col + e] : 0.f);
    if (out_type == BITA_F32) {
        float *p = (float *)out + (int64_t)row * ldo + col;
        if (col + 4 <= n) *reinterpret_cast<Words4 *>(p) = Words4{{v[0], v[1], v[2], v[3]}};
        else
            for (int e = 0; e < 3; e++)
                if (col + e < n) p[e] = v[e];
    } else {
        uint16_t *p = (uint16_t *)out + (int64_t)row * ldo + col, h[4];
#pragma unroll
        for (int e = 0; e < 4; e++) h[e] = __builtin_bit_cast(uint16_t, (__bf16)v[e]);
        if (col + 4 <= n) *reinterpret_cast<Halves4 *>(p) = Halves4{{h[0], h[1], h[2], h[3]}};
        else
            for (int e = 0; e < 3; e++)
                if (col + e < n) p[e] = h[e];
    }
}

// V neighbouring columns of one row (16 bytes), with their scales
struct __attribute__((packed, aligned(2))) Halves8 { uint32_t w[4]; };
template <int V>
__device__ __forceinline__ void store_row(float *out, int64_t ldo, int row, int64_t col, int64_t n, const int sum[V], float sa, const float scale[V]) {
    float *p = out + (int64_t)row * ldo + col, v[V];
#pragma unroll
    for (int e = 0; e < V; e++) v[e] = (float)sum[e] * sa * scale[e];
    if (col + V <= n) {
        *reinterpret_cast<Words4 *>(p) = Words4{{v[0], v[1], v[2], v[3]}};
        return;
    }
#pragma unroll
    for (int e = 0; e < V; e++)
        if (col + e < n) p[e] = v[e];
}
template <int V>
__device__ __forceinline__ void store_row(int *out, int64_t ldo, int row, int64_t col, int64_t, const int sum[V], float, const float *) {      // (whole tiles: no end inside)
    *reinterpret_cast<i32x4 *>(out + (int64_t)row * ldo + col) = i32x4{sum[0], sum[1], sum[2], sum[3]};
}
template <int V>
__device__ __forceinline__ void store_row(uint16_t *out, int64_t ldo, int row, int64_t col, int64_t n, const int sum[V], float sa, const float scale[V]) {
    uint16_t *p = out + (int64_t)row * ldo + col, h[V];
#pragma unroll
    for (int e = 0; e < V; e++) h[e] = __builtin_bit_cast(uint16_t, (__bf16)((float)sum[e] * sa * scale[e]));
    if (col + V <= n) {
        Halves8 q;
#pragma unroll
        for (int e = 0; e < V / 2; e++) q.w[e] = h[2 * e] | (uint32_t)h[2 * e + 1] << 16;
        *reinterpret_cast<Halves8 *>(p) = q;
        return;
    }
#pragma unroll
    for (int e = 0; e < V; e++)
        if (col + e < n) p[e] = h[e];
}

// Few rows, one pass over the weights.  A workgroup has MT tiles of 16 rows and WN of 16 columns; KG groups of WN waves share the
// k-steps of a stage (512 k) and are summed through LDS at the end.  A weight block is one matrix operand (16 columns x 64 k, lane l
// column l % 16, k 16 (l / 16)) and goes straight to the registers of the one wave that multiplies it.  Activations pass through two
// LDS buffers of a stage: every load takes two rows of 512 bytes (16 rows of 64 bytes, the operand's own shape, arrive at 34 GB/s
// a CU instead of 94), and piece p of row x lies at p ^ (x % 16), so that the 16 rows of an operand are 16 bank groups.
// What bounds it: a CU has about 32 KB of loads in flight, answered in order, which at the latency of HBM is 50 to 60 GB/s, rows
// and weights together; deeper prefetch (4 stages ahead) measured the same, a descriptor that starts each workgroup at another
// stage too.  Cutting so that a CU's rows and weights are few is plan_q8's business.  One row of 8192 x 28672: 36 us, 6.4 TB/s;
// 68 rows of 22016 x 4096 22 us (the wave that loads its own rows: 42), of 4096 x 4096 9.9.
template <int MT, int WN, int KG, int P>
__global__ __launch_bounds__(WN * KG * 64) void gemm_q8_skinny_kernel(const int8_t *__restrict__ a, int64_t lda, const i32x4 *__restrict__ w, int m, int k_steps,
                                                             int k16, int64_t n, const float *__restrict__ sa, const float *__restrict__ sw,
                                                             void *__restrict__ out, int64_t ldo, int out_type, int split_steps, int *__restrict__ part) {
    constexpr int SK = 8, WAVES = WN * KG, SW = SK / KG;                         // k-steps of a stage, of a wave in it
    constexpr int ROWS = 16 * MT, STAGE = ROWS * 32, NL = STAGE / 64, AL = (NL + WAVES - 1) / WAVES;   // 16-byte pieces of a stage; its loads, a wave's
    extern __shared__ __attribute__((aligned(16))) i32x4 lds[];                  // [2][ROWS][32], then [KG][MT * WN][64]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kg = wave / WN, wn = wave % WN, r = lane & 15, c = lane >> 4;
    const int64_t n_tiles = (n + 15) >> 4, tile = (int64_t)blockIdx.x * WN + wn;
    const int m0 = blockIdx.y * ROWS, first = blockIdx.z * split_steps, last = min(k_steps, first + split_steps), stages = (last - first + SK - 1) / SK;
    // (offsets out of the descriptor's range read zeros and move nothing: rows and columns past the end, stages past the last)
    constexpr uint32_t NOWHERE = 0xFFFFFFF0u;
    const int8_t *ab = a + (int64_t)m0 * lda;
    const int rows = min(m - m0, ROWS), k_end = min(k16, last * 64);
    const __amdgpu_buffer_rsrc_t a_rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)ab, 0, (uint32_t)((rows - 1) * lda + k16), 0x00027000);
    uint32_t a_row[AL];
    int piece[AL];
#pragma unroll
    for (int i = 0; i < AL; i++) {
        const int x = 2 * (i * WAVES + wave) + (lane >> 5);
        a_row[i] = x < rows ? (uint32_t)(x * lda) : NOWHERE;                 // (loads past the last row of the tile: none)
        piece[i] = ((lane & 31) ^ (x & 15)) * 16;
    }
    const i32x4 *wt = w + min(tile, n_tiles - 1) * 128;
    const uint32_t w_bytes = tile < n_tiles ? 2048 : 0;
    i32x4 ra[P][AL], rb[P][SW], acc[MT];
    auto fetch_a = [&](int set, int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < AL; i++) {
            const int col = (first + t * SK) * 64 + piece[i];
            ra[set][i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(a_rsrc, col < k_end && a_row[i] != NOWHERE ? a_row[i] + col : NOWHERE, 0, 0));
        }
    };
    auto fetch_b = [&](int set, int t, int s) __attribute__((always_inline)) {
        const int ks = first + t * SK + kg * SW + s;
        const __amdgpu_buffer_rsrc_t rsrc =
            __builtin_amdgcn_make_buffer_rsrc((void *)(wt + ((int64_t)(ks >> 1) * n_tiles * 2 + (ks & 1)) * 64), 0, ks < last ? w_bytes : 0, 0x00027000);
        rb[set][s] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane * 16, 0, /* nt */ 2));
    };
    i32x4 fa[2][MT];
    auto read_a = [&](int buf, int s) __attribute__((always_inline)) {
        const int at = buf * STAGE + r * 32 + (((kg * SW + s) * 4 + c) ^ r);
#pragma unroll
        for (int i = 0; i < MT; i++) fa[s & 1][i] = lds[at + i * 512];
    };
    auto put_a = [&](int buf, int set) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < AL; i++)
            if ((i + 1) * WAVES <= NL || i * WAVES + wave < NL) lds[buf * STAGE + (i * WAVES + wave) * 64 + lane] = ra[set][i];
    };
    auto barrier = [&]() __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);                                  // lgkmcnt(0): this wave's LDS writes and reads are done
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < MT; i++) acc[i] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < P; u++) {
        fetch_a(u, u);
#pragma unroll
        for (int s = 0; s < SW; s++) fetch_b(u, u, s);
        __builtin_amdgcn_sched_barrier(0);
    }
    put_a(0, 0);
    fetch_a(0, P);
    __builtin_amdgcn_sched_barrier(0);
    barrier();
    for (int t = 0; t < stages; t += P) {
#pragma unroll
        for (int u = 0; u < P; u++) {
            read_a((t + u) & 1, 0);
#pragma unroll
            for (int s = 0; s < SW; s++) {
                if (s + 1 < SW) read_a((t + u) & 1, s + 1);
                __builtin_amdgcn_sched_barrier(0);
                if (t + u < stages) {
#pragma unroll
                    for (int i = 0; i < MT; i++) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(rb[u][s], fa[s & 1][i], acc[i], 0, 0, 0);
                }
                fetch_b(u, t + u + P, s);
                __builtin_amdgcn_sched_barrier(0);
            }
            put_a((t + u + 1) & 1, (u + 1) % P);                                 // (its buffer was read before the last barrier)
            fetch_a((u + 1) % P, t + u + 1 + P);
            __builtin_amdgcn_sched_barrier(0);
            barrier();
        }
    }
    // lane l of a tile's sums: row l % 16, columns 4 (l / 16) .. + 3
    auto store = [&](int i, int64_t tile, i32x4 v) __attribute__((always_inline)) {
        const int row = m0 + 16 * i + r;
        const int64_t col = tile * 16 + 4 * c;
        if (row >= m || col >= n) return;
        if (part)                                                            // (whole tiles of columns: the last one's padding is written too)
            *reinterpret_cast<i32x4 *>(part + ((int64_t)blockIdx.z * m + row) * (n_tiles * 16) + col) = v;
        else
            store4(out, out_type, ldo, row, col, n, v, sa[row], sw);
    };
    if constexpr (KG == 1) {
#pragma unroll
        for (int i = 0; i < MT; i++) store(i, tile, acc[i]);
    } else {
        constexpr int TILES = MT * WN;
#pragma unroll
        for (int i = 0; i < MT; i++) lds[(kg * TILES + i * WN + wn) * 64 + lane] = acc[i];
        __syncthreads();
        for (int f = wave; f < TILES; f += WAVES) {
            i32x4 sum = lds[f * 64 + lane];
#pragma unroll
            for (int g = 1; g < KG; g++) sum += lds[(g * TILES + f) * 64 + lane];
            store(f / WN, (int64_t)blockIdx.x * WN + f % WN, sum);
        }
    }
}

// Sums of the k splits, scaled and stored: a thread has four columns of a row (ld4: a row's groups of four).
__global__ __launch_bounds__(256) void gemm_q8_reduce_kernel(const i32x4 *__restrict__ part, int splits, int m, int64_t n, uint32_t ld4, const float *__restrict__ sa,
                                                             const float *__restrict__ sw, void *__restrict__ out, int64_t ldo, int out_type) {
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = at / ld4, col = (at - row * ld4) * 4;
    if (row >= (uint32_t)m || col >= n) return;
    const int64_t step = (int64_t)m * ld4;
    i32x4 q[8], sum = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < 8; s++) q[s] = part[at + min(s, splits - 1) * step];      // (requested together; those past the last are left out)
#pragma unroll
    for (int s = 0; s < 8; s++)
        if (s < splits) sum += q[s];
    store4(out, out_type, ldo, row, col, n, sum, sa[row], sw);
}

// Many rows: tiles of 32 MF WM rows and 32 NF WN columns, WM x WN waves of MF x NF matrix tiles of 32 x 32 each, both operands
// through two LDS buffers of 128 k: rows of 128 bytes with piece p of row x at p ^ (x % 8), weight blocks as they are packed (the
// stage's are one run of memory).  Each stage's loads are spread over its matrix instructions, two stages ahead of their use.
// What bounds 256 x 256 tiles (4096 rows x 57344 x 8192, 1.76 ms, 2190 TOP/s; the library's 8192^3 2400): the matrix instructions
// and the stores take 1.30 ms (at the clock that the card holds under them), LDS reads 0.19 more, LDS writes 0.13, loads 0.25.  Weights
// straight to the registers of the WM waves that use them: 1.90 ms against 1.85 at the time; four waves of 128 x 128: 2.01.
template <int MF, int NF, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void gemm_q8_tile_kernel(
    const int8_t *__restrict__ a, int64_t lda, const i32x4 *__restrict__ w, int m, int k_pairs, int k16, int64_t n, int m_blocks, int n_blocks,
    const float *__restrict__ sa, const float *__restrict__ sw, void *__restrict__ out, int64_t ldo, int out_type, int split_pairs, int *__restrict__ part) {
    typedef __attribute__((ext_vector_type(16))) int i32x16;
    constexpr int WAVES = WM * WN, BM = 32 * MF * WM, AW = (BM / 8 + WAVES - 1) / WAVES;           // loads of 8 rows x 128 bytes, of a wave
    constexpr int BN = 32 * NF * WN, BW = (BN / 8 + WAVES - 1) / WAVES, LW = AW + BW;              // 1 KiB loads of weights, of a wave; of both
    extern __shared__ __attribute__((aligned(16))) i32x4 lds[];                      // [2][BM rows: [piece ^ row % 8] | BN / 16 blocks of 2 KiB]
    constexpr int STAGE = (BM + BN) * 8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    // tiles of one XCD (workgroups id % 8) are neighbours: groups of 8 row blocks, column block by column block
    const int total = m_blocks * n_blocks, per_xcd = (total + 7) / 8;
    const int id = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (id >= total || (int)(blockIdx.x >> 3) >= per_xcd) return;
    const int group = id / (8 * n_blocks), in_group = id - group * 8 * n_blocks, tall = min(8, m_blocks - group * 8);
    const int nb = in_group / tall, mb = group * 8 + in_group - nb * tall;
    const int m0 = mb * BM, first = blockIdx.y * split_pairs, pairs = min(k_pairs - first, split_pairs), k_end = min(k16, (first + pairs) * 128);
    const int64_t n_tiles = (n + 15) >> 4, tile0 = (int64_t)nb * (BN / 16) + wn * 2 * NF;
    // (offsets out of the descriptor's range read zeros and move nothing)
    constexpr uint32_t NOWHERE = 0xFFFFFFF0u;
    const int rows = min(m - m0, BM), piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const __amdgpu_buffer_rsrc_t a_rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(a + (int64_t)m0 * lda), 0, (uint32_t)((rows - 1) * lda + k16), 0x00027000);
    uint32_t a_row[AW];
#pragma unroll
    for (int i = 0; i < AW; i++) {
        const int x = 8 * (i * WAVES + wave) + (lane >> 3);
        a_row[i] = x < rows ? (uint32_t)(x * lda) + piece : NOWHERE;
    }
    // operand of a 32 x 32 x 32 instruction: lane l holds row l % 32, 16 k's from 16 (l / 32)
    const int half = lane >> 5, r = lane & 31;
    const i32x4 *wt = w + (int64_t)nb * (BN / 16) * 128;
    const uint32_t w_bytes = (uint32_t)min((int64_t)(BN / 16), n_tiles - (int64_t)nb * (BN / 16)) * 2048;
    const int a_at = (wm * MF * 32 + r) * 8, b_at = BM * 8 + (wn * NF * 2 + (r >> 4)) * 128 + half * 16 + (lane & 15);
    i32x4 st[LW], fa[2][MF], fb[2][NF];
    i32x16 acc[MF][NF];
    // the loads of a stage, one by one: the wave's rows of activations, then its pieces of the stage's weight blocks (one run of memory)
    auto fetch = [&](int i, int t) __attribute__((always_inline)) {
        if (i < AW) {
            const int col = (first + t) * 128;
            st[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(a_rsrc, col + piece < k_end && a_row[i < AW ? i : 0] != NOWHERE ? a_row[i < AW ? i : 0] + col : NOWHERE, 0, 0));
        } else {
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(wt + (int64_t)(first + t) * n_tiles * 128), 0, t < pairs ? w_bytes : 0, 0x00027000);
            st[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (i - AW) * WAVES + wave < BN / 8 ? ((i - AW) * WAVES + wave) * 1024 + lane * 16 : NOWHERE, 0, 0));
        }
    };
    auto put = [&](int i, int buf) __attribute__((always_inline)) {
        const int p = i < AW ? i * WAVES + wave : (i - AW) * WAVES + wave;
        if (p < (i < AW ? BM : BN) / 8) lds[buf * STAGE + (i < AW ? 0 : BM * 8) + p * 64 + lane] = st[i];
    };
    auto read = [&](int buf, int q) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NF; j++) fb[q & 1][j] = lds[buf * STAGE + b_at + j * 256 + q * 32];
#pragma unroll
        for (int i = 0; i < MF; i++) fa[q & 1][i] = lds[buf * STAGE + a_at + i * 256 + ((2 * q + half) ^ (r & 7))];
    };
    auto barrier = [&]() __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);                                  // lgkmcnt(0): this wave's LDS writes and reads are done
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < MF; i++)
#pragma unroll
        for (int j = 0; j < NF; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0;
#pragma unroll
    for (int i = 0; i < LW; i++) fetch(i, 0);
#pragma unroll
    for (int i = 0; i < LW; i++) {
        put(i, 0);
        fetch(i, 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    barrier();
    for (int t = 0; t < pairs; t++) {
        const int buf = t & 1;
        read(buf, 0);
#pragma unroll
        for (int q = 0; q < 4; q++) {
            if (q < 3) read(buf, q + 1);
            // a third of the next stage goes to the other buffer (read before the last barrier), and the one after it is asked for
            if (q > 0) {
#pragma unroll
                for (int i = (q - 1) * LW / 3; i < q * LW / 3; i++) {
                    put(i, buf ^ 1);
                    fetch(i, t + 2);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < MF; i++)
#pragma unroll
                for (int j = 0; j < NF; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[q & 1][j], fa[q & 1][i], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        barrier();
    }
    // Sums leave as whole row segments: lane l of a tile has row l % 32 and, as value e, column 8 (e / 4) + 4 (l / 32) + e % 4, 16 bytes of each of
    // 32 rows a store; so a wave turns 32 rows at a time in LDS of its own (16 bytes more a row: rows start in different banks).  Straight from the
    // registers 4096 rows of 22016 x 4096 in bf16 took 100 us longer than without stores.
    constexpr int COLS = 32 * NF, LD = COLS / 4 + 1;                                  // in 16-byte pieces
    static_assert(WAVES * 32 * LD <= 2 * STAGE && (NF & (NF - 1)) == 0, "the epilogue's rows fit the stages, its lanes divide a wave");
    i32x4 *own = lds + wave * 32 * LD;
    // between lanes' stores there and other lanes' reads, and before the next stores: a wave's LDS operations keep their order, which the compiler
    // has to keep too (to it a lane's store and its reads are of places that may be told apart); no instruction
    auto turned = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    auto leave = [&](auto *o, int64_t ldo, int64_t n) __attribute__((always_inline)) {
        constexpr int V = 16 / (int)sizeof(*o), LANES = COLS / V, ROWS = 64 / LANES;  // columns of a lane, lanes of a row, rows a store
        const int c = lane % LANES;
        const int64_t col = tile0 * 16 + c * V;
        float scale[V];
#pragma unroll
        for (int e = 0; e < V; e++) scale[e] = !part && col + e < n ? sw[col + e] : 0.f;
#pragma unroll
        for (int i = 0; i < MF; i++) {
            const int first = m0 + (wm * MF + i) * 32;
            if (first >= m) break;
#pragma unroll
            for (int j = 0; j < NF; j++)
#pragma unroll
                for (int e = 0; e < 4; e++)
                    own[r * LD + j * 8 + 2 * e + half] = i32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
            turned();
#pragma unroll
            for (int x = 0; x < 32; x += ROWS) {
                const int in = x + lane / LANES, row = first + in;
                int sum[V];
#pragma unroll
                for (int e = 0; e < V / 4; e++) {
                    const i32x4 q = own[in * LD + c * (V / 4) + e];
                    sum[4 * e] = q[0]; sum[4 * e + 1] = q[1]; sum[4 * e + 2] = q[2]; sum[4 * e + 3] = q[3];
                }
                if (row < m && col < n) store_row<V>(o, ldo, row, col, n, sum, sa[row], scale);
            }
            turned();
        }
    };
    if (part) leave(part + (int64_t)blockIdx.y * m * n_tiles * 16, n_tiles * 16, n_tiles * 16);
    else if (out_type == BITA_F32) leave((float *)out, ldo, n);
    else leave((uint16_t *)out, ldo, n);
}

// ---------------------------------------------------------------------------------------
struct GemmQ8 {
    const int8_t *a; int64_t lda; const float *sa; int m, k_pairs, k16; const i32x4 *w; const float *sw; int64_t n;
    void *out; int out_type; int64_t ldo; int *part; hipStream_t s;
};
// How a product is cut.  form < SKINNY: a tile kernel; else weight tiles side by side in a workgroup of the skinny kernel, whose
// workgroups have mt row tiles each; splits of k (at most 8), of split_steps k-steps each.
enum { SKINNY = 16 };
struct PlanQ8 { int form, mt, splits, split_steps; };

// Tile kernels: rows and columns of a workgroup, and the time of 128 k of one, us (1024 rows x 4096 x 4096 in one round, 288 x 128 at 272 rows of
// 22016 x 4096: 49 us, with 160 x 256 57, 96 x 192 53).  The times follow the bytes of a stage, 32 to 42 GB/s a CU: half as many waves of
// twice the columns, with fewer LDS reads, are no faster (160 x 256 by four waves 58).
struct TileForm { int rows, cols; float stage; };
static const TileForm TILE_FORMS[] = {{256, 256, 2.06f}, {160, 256, 1.53f}, {128, 256, 1.16f}, {128, 128, 0.82f}, {96, 192, 0.90f}, {288, 128, 1.36f}};
static const int SKINNY_WIDE[] = {1, 2, 3, 4, 6, 8};
#define SKINNY_MAX_MT 9

// Whichever form promises the least time.  What the estimates rest on (measured):
//  * a CU has about 32 KB of vector loads in flight and gets them in order: 56 GB/s of weights and activations together where the
//    weights come from HBM, whatever is behind its L1; hence few rows are cut so that all 256 CUs work and a workgroup's rows,
//    which every workgroup reads, are amortised over many columns, by splitting k if need be;
//  * the few-rows kernel reads LDS once for each matrix instruction: 0.012 us a stage for each of its tiles of 16 x 16;
//  * weights alone arrive at 6.3 TB/s; a launch costs 3.5 us and 1.5 more for each further round of workgroups, a second one (the splits' sums) 3 us and its traffic.
// With every form and split of 148 products of 1 to 1024 rows timed, its choices are 1.0 % slower than the best in the mean and 15 % at most.
static PlanQ8 plan_q8(int m, int64_t n, int k_pairs) {
    const int64_t n_tiles = (n + 15) / 16;
    const int stages = (k_pairs + 3) / 4;
    PlanQ8 best = {};
    double best_us = 1e30;
    const double weights_us = 2048.0 * n_tiles * k_pairs / 6.3e6;
    const auto sums_us = [&](int splits) { return splits > 1 ? 3 + 8.0 * splits * m * (16.0 * n_tiles) / 4.5e6 : 0.0; };
    const int forms = m > 16 ? (int)(sizeof(TILE_FORMS) / sizeof(TILE_FORMS[0])) : 0;       // (16 rows of 57344 x 8192: 75 us, in tiles of 128 80)
    for (int f = 0; f < forms; f++)
        for (int splits = 1; splits <= 8 && (splits == 1 || splits * 8 <= k_pairs); splits++) {
            const TileForm &t = TILE_FORMS[f];
            const int per = (k_pairs + splits - 1) / splits;
            if ((k_pairs + per - 1) / per != splits) continue;
            const double tiles = (double)(((int64_t)m + t.rows - 1) / t.rows) * (double)((n + t.cols - 1) / t.cols);
            if (splits > 1 && tiles * splits > 512) break;                      // (enough workgroups as it is)
            const double us = 5 + fmax(ceil(tiles * splits / 256) * per * t.stage, weights_us) + sums_us(splits);
            if (us < best_us) { best_us = us; best = {f, 0, splits, 2 * per}; }
        }
    if (m > 2 * SKINNY_MAX_MT * 16) return best;
    const int mt_all = (m + 15) / 16, blocks = (mt_all + SKINNY_MAX_MT - 1) / SKINNY_MAX_MT, mt = (mt_all + blocks - 1) / blocks;
    for (int wide : SKINNY_WIDE) {
        if (wide == 6 && mt == 9) continue;                                  // (its registers do not suffice)
        for (int splits = 1; splits <= 8 && (splits == 1 || splits * 4 <= stages); splits++) {
            const int per = (stages + splits - 1) / splits, s = (stages + per - 1) / per;
            if (s != splits) continue;
            const double groups = (double)((n_tiles + wide - 1) / wide) * blocks * splits, rounds = ceil(groups / 256);
            const double bytes = 512.0 * ((m + blocks - 1) / blocks + 16 * wide);
            const double stage = fmax(0.34, bytes / 56e3 + 0.012 * mt * wide);
            const double us = 2 + 1.5 * rounds + fmax(rounds * per * stage, weights_us) + sums_us(splits);
            if (us < best_us) { best_us = us; best = {SKINNY + wide, mt, splits, 8 * per}; }
        }
    }
    return best;
}

// More LDS than the default limit has to be asked for, once for each kernel and device.
struct LdsLimit { std::atomic<uint64_t> devices{0}; };
static void raise_lds_limit(LdsLimit &done, const void *kernel, int bytes) {
    int dev = 0;
    if (bytes <= 65536 || hipGetDevice(&dev) != hipSuccess) return;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (bit && (done.devices.load(std::memory_order_relaxed) & bit)) return;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess) done.devices.fetch_or(bit, std::memory_order_relaxed);
}

template <int MT, int WN, int KG, int P>
static void launch_skinny(const GemmQ8 &g, const PlanQ8 &p) {
    constexpr int STAGES = 2 * MT * 8192, MERGE = KG > 1 ? KG * WN * MT * 1024 : 0, SMEM = STAGES > MERGE ? STAGES : MERGE;
    static LdsLimit limit;
    raise_lds_limit(limit, (const void *)gemm_q8_skinny_kernel<MT, WN, KG, P>, SMEM);
    const int64_t tiles = (g.n + 15) / 16;
    hipLaunchKernelGGL((gemm_q8_skinny_kernel<MT, WN, KG, P>), dim3((unsigned)((tiles + WN - 1) / WN), (unsigned)((g.m + 16 * MT - 1) / (16 * MT)), p.splits),
                       dim3(WN * KG * 64), SMEM, g.s, g.a, g.lda, g.w, g.m, 2 * g.k_pairs, g.k16, g.n, g.sa, g.sw, g.out, g.ldo, g.out_type, p.split_steps,
                       p.splits > 1 ? g.part : nullptr);
}
static void launch_reduce(const GemmQ8 &g, const PlanQ8 &p) {
    const uint32_t ld4 = (uint32_t)((g.n + 15) / 16 * 4);
    hipLaunchKernelGGL(gemm_q8_reduce_kernel, dim3((unsigned)(((uint64_t)g.m * ld4 + 255) / 256)), dim3(256), 0, g.s, (const i32x4 *)g.part, p.splits, g.m, g.n,
                       ld4, g.sa, g.sw, g.out, g.ldo, g.out_type);
}
template <int MF, int NF, int WM, int WN>
static void launch_tile(const GemmQ8 &g, const PlanQ8 &p) {
    constexpr int BM = 32 * MF * WM, BN = 32 * NF * WN, SMEM = 2 * (BM + BN) * 128;
    const int m_blocks = (int)(((int64_t)g.m + BM - 1) / BM), n_blocks = (int)((g.n + BN - 1) / BN), total = m_blocks * n_blocks;
    static LdsLimit limit;
    raise_lds_limit(limit, (const void *)gemm_q8_tile_kernel<MF, NF, WM, WN>, SMEM);
    hipLaunchKernelGGL((gemm_q8_tile_kernel<MF, NF, WM, WN>), dim3((unsigned)((total + 7) / 8 * 8), p.splits), dim3(WM * WN * 64), SMEM, g.s, g.a, g.lda, g.w, g.m,
                       g.k_pairs, g.k16, g.n, m_blocks, n_blocks, g.sa, g.sw, g.out, g.ldo, g.out_type, p.split_steps / 2, p.splits > 1 ? g.part : nullptr);
}
// waves that share k where a workgroup has few columns; k two stages ahead where a stage is short
template <int MT>
static void launch_skinny_mt(const GemmQ8 &g, const PlanQ8 &p) {
    switch (p.form - SKINNY) {
        case 1: return launch_skinny<MT, 1, 8, 2>(g, p);
        case 2: return launch_skinny<MT, 2, 4, 2>(g, p);
        case 3: return launch_skinny<MT, 3, MT <= 5 ? 4 : 2, 1>(g, p);       // (12 waves have 168 registers each)
        case 4: return launch_skinny<MT, 4, 2, 1>(g, p);
        case 6: return launch_skinny<MT < 9 ? MT : 8, 6, MT <= 7 ? 2 : 1, 1>(g, p);
        default: return launch_skinny<MT, 8, 1, 1>(g, p);
    }
}
static void launch_gemm_q8(const GemmQ8 &g, const PlanQ8 &p) {
    if (p.form < SKINNY) {
        switch (p.form) {
            case 0: return launch_tile<4, 2, 2, 4>(g, p);
            case 1: return launch_tile<5, 1, 1, 8>(g, p);
            case 2: return launch_tile<2, 2, 2, 4>(g, p);
            case 3: return launch_tile<2, 1, 2, 4>(g, p);
            case 4: return launch_tile<3, 1, 1, 6>(g, p);
            default: return launch_tile<3, 2, 3, 2>(g, p);
        }
    }
    switch (p.mt) {
        case 1: return launch_skinny_mt<1>(g, p);
        case 2: return launch_skinny_mt<2>(g, p);
        case 3: return launch_skinny_mt<3>(g, p);
        case 4: return launch_skinny_mt<4>(g, p);
        case 5: return launch_skinny_mt<5>(g, p);
        case 6: return launch_skinny_mt<6>(g, p);
        case 7: return launch_skinny_mt<7>(g, p);
        case 8: return launch_skinny_mt<8>(g, p);
        default: return launch_skinny_mt<9>(g, p);
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
    const int64_t tiles = (n_rows + 15) / 16, total = (dst_total_rows + 15) / 16, last = (int64_t)((uint64_t)dst_tile0 + (uint64_t)(tiles - 1) * (uint64_t)dst_tile_stride);
    if (dst_tile0 >= total || (tiles > 1 && dst_tile_stride >= total) || last >= total)      // (the first two: `last` did not wrap)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_pack_weight_q8: source tiles do not fit %lld destination rows", (long long)dst_total_rows);
    if (n_rows % 16 && last != total - 1)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_pack_weight_q8: %lld rows end inside a tile that is not the destination's last", (long long)n_rows);
    if (k > BITA_Q8_MAX_K || n_rows > BITA_Q8_MAX_N)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_pack_weight_q8: %lld rows of %lld", (long long)n_rows, (long long)k);
    hipLaunchKernelGGL(pack_q8_kernel, dim3((unsigned)tiles, (unsigned)min((int64_t)8, (k + 255) / 256)), dim3(256), 0, (hipStream_t)stream, d_src, n_rows,
                       k, ld, (uint4 *)d_dst, dst_tile0, dst_tile_stride, total);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}

static size_t plan_bytes(const PlanQ8 &p, int m, int64_t n) { return p.splits > 1 ? (size_t)p.splits * m * (size_t)((n + 15) / 16 * 16) * 4 : 0; }

extern "C" size_t bita_gemm_q8_workspace_bytes(int32_t m_rows, int64_t n_rows, int64_t k) {
    if (m_rows <= 0 || n_rows <= 0 || k <= 0 || k > BITA_Q8_MAX_K || n_rows > BITA_Q8_MAX_N) return 0;
    return plan_bytes(plan_q8(m_rows, n_rows, (int)((k + 127) / 128)), m_rows, n_rows);
}

extern "C" int bita_gemm_q8_plan_info(int32_t m_rows, int64_t n_rows, int64_t k, int32_t *out4) {
    if (!out4 || m_rows <= 0 || n_rows <= 0 || k <= 0 || k > BITA_Q8_MAX_K || n_rows > BITA_Q8_MAX_N)
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_gemm_q8_plan_info: bad argument");
    const PlanQ8 p = plan_q8(m_rows, n_rows, (int)((k + 127) / 128));
    const bool skinny = p.form >= SKINNY;
    out4[0] = skinny ? 16 * p.mt : TILE_FORMS[p.form].rows;
    out4[1] = skinny ? 16 * (p.form - SKINNY) : TILE_FORMS[p.form].cols;
    out4[2] = p.splits;
    out4[3] = skinny;
    return BITA_OK;
}

int gemm_q8(const int8_t *d_a, int64_t lda, const float *d_a_scale, int32_t m_rows, int64_t k, const void *d_w_packed, const float *d_w_scale, int64_t n_rows,
            void *d_ws, size_t ws_bytes, void *d_out, int32_t out_type, int64_t ldo, SumsQ8 *left, hipStream_t s) {
    if (!d_a || !d_a_scale || !d_w_packed || !d_w_scale || !d_out || m_rows <= 0 || k <= 0 || n_rows <= 0 || ldo < n_rows ||
        (out_type != BITA_F32 && out_type != BITA_BF16))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_gemm_q8: bad argument");
    if ((uintptr_t)d_a % 16 || (uintptr_t)d_w_packed % 16 || lda % 16 || (m_rows > 1 && lda < k) || (uintptr_t)d_out % (out_type == BITA_BF16 ? 2 : 4))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_gemm_q8: d_a, d_w_packed and lda have to be multiples of 16, lda at least k");
    if (k > BITA_Q8_MAX_K || lda > BITA_Q8_MAX_LD || n_rows > BITA_Q8_MAX_N)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_gemm_q8: k %lld, lda %lld, n_rows %lld, at most %d, %d and %d", (long long)k, (long long)lda,
                              (long long)n_rows, BITA_Q8_MAX_K, BITA_Q8_MAX_LD, BITA_Q8_MAX_N);
    const int k_pairs = (int)((k + 127) / 128), k16 = (int)((k + 15) / 16 * 16);
    const PlanQ8 p = plan_q8(m_rows, n_rows, k_pairs);
    const size_t need = plan_bytes(p, m_rows, n_rows);
    if (need && (!d_ws || ws_bytes < need || (uintptr_t)d_ws % 16))
        return bita_set_error(BITA_ERR_CAPACITY, "bita_gemm_q8: workspace %zu < %zu bytes, or not a multiple of 16", d_ws ? ws_bytes : (size_t)0, need);
    const GemmQ8 g = {d_a, lda, d_a_scale, m_rows, k_pairs, k16, (const i32x4 *)d_w_packed, d_w_scale, n_rows, d_out, out_type, ldo, (int *)d_ws, s};
    launch_gemm_q8(g, p);
    if (left) *left = p.splits > 1 ? SumsQ8{g.part, p.splits, d_a_scale, d_w_scale} : SumsQ8{};
    else if (p.splits > 1) launch_reduce(g, p);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}

extern "C" int bita_gemm_q8(const int8_t *d_a, int64_t lda, const float *d_a_scale, int32_t m_rows, int64_t k, const void *d_w_packed,
                            const float *d_w_scale, int64_t n_rows, void *d_ws, size_t ws_bytes, void *d_out, int32_t out_type, int64_t ldo, void *stream) {
    return gemm_q8(d_a, lda, d_a_scale, m_rows, k, d_w_packed, d_w_scale, n_rows, d_ws, ws_bytes, d_out, out_type, ldo, nullptr, (hipStream_t)stream);
}
