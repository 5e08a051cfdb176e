// The 4- and 8-bit K/V cache: rows rounded to microscaled blocks as they are written, and read back.
//
// A thread holds 8 neighbouring values of a head, four threads a block: its largest magnitude is an integer maximum over the four
// (the fp32 bits without the sign are in the order of the magnitudes, infinities and NaN above all), its exponent comes from those
// bits, and the conversion instructions divide by the power of two and round once.  A workgroup takes 16 or 32 rows of one head,
// which are neighbours in the cache.  Both directions move little more than the tensors themselves, which is what bounds them: 8192 packed fp32 rows of 40 heads of 128
// to 4 bits, 380 MB, 79 us alone (4.8 TB/s) and 88 behind other work, back to bf16, 212 MB, 40.5 (5.2 TB/s); 24 296 slots of 8 heads from 8 bits, 151 MB, 24.5 us.  4 rows of 4
// heads a workgroup write in the same time, reads past the caches in 88 us.  A step's 22 rows: 3.0 us there, 2.8 back.
#include "mx.h"

#define MX_THREADS 256
#define MX_MAX_ROWS (1 << 27)           // of a call and sequence: a grid holds 2^32 threads along x

// The sequence of a row of the packed axis: the last one that starts at or before it (`batch`: the row is behind all of them; 0 also where it is before
// all).  64 starts are looked at in a step, and the 64th part they leave in the next.
__device__ __forceinline__ int packed_sequence(const int32_t *__restrict__ cu, int batch, int row) {
    const int lane = threadIdx.x & 63;
    int b = 0, n = batch + 1;                                   // it is among n from b on
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const uint64_t before = __builtin_amdgcn_ballot_w64(at < n && cu[b + min(at, n - 1)] <= row);
        if (before == 0) break;
        const int last = 63 - __builtin_clzll(before);
        b += last * step;
        n = min(step, n - last * step);
    }
    return b;
}

template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

template <int HD, int BITS>
__device__ __forceinline__ void put_block(float (&v)[8], unsigned char *codes, uint8_t *scales, int64_t row, int part) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const uint32_t byte = mx_scale_byte<BITS>(top);
    if (byte == 255) {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = 0.f;
    }
    const float scale = byte == 255 ? 1.f : mx_scale(byte);
    if (row < 0) return;
    unsigned char *dst = codes + row * (HD * BITS / 8) + part * BITS;
    if constexpr (BITS == 4) *reinterpret_cast<uint32_t *>(dst) = mx_encode4(v, scale);
    else *reinterpret_cast<uint2 *>(dst) = mx_encode8(v, scale);
    if ((part & 3) == 0) scales[row * (HD / 32) + (part >> 2)] = (uint8_t)byte;
}

template <typename T, int HD, int BITS>
__global__ __launch_bounds__(MX_THREADS) void kv_write_mx_kernel(KvMx kv, const T *__restrict__ k, MxRows ks, const T *__restrict__ v, MxRows vs, int n_rows,
                                                                 const int32_t *__restrict__ start,
                                                                 const int32_t *__restrict__ count, const int32_t *__restrict__ path, int path_stride,
                                                                 const int32_t *__restrict__ cu) {
    constexpr int PARTS = HD / 8, ROWS = MX_THREADS / PARTS;
    const int part = threadIdx.x % PARTS, tile = blockIdx.x / kv.Hkv, h = blockIdx.x - tile * kv.Hkv;  // (a row's heads are neighbours where rows are packed)
    int i = tile * ROWS + threadIdx.x / PARTS, b = cu ? 0 : blockIdx.y;
    const int entries = path ? path_stride : n_rows, at = min(i, entries - 1);
    const int src = min(max(path ? path[(int64_t)b * path_stride + at] : at, 0), n_rows - 1);
    // the rows are on their way while their place is looked for
    float x[8], y[8];
    load8(k + ks.at(b, h, src) + part * 8, x);
    load8(v + vs.at(b, h, src) + part * 8, y);
    bool ok = i < entries;
    if (cu) {
        b = packed_sequence(cu, kv.batch, tile * ROWS);
        while (b < kv.batch && cu[b + 1] <= src) b++;
        ok = ok && b < kv.batch;
        b = min(b, kv.batch - 1);
        i = src - cu[b];
    }
    ok = ok && i >= 0 && (!count || i < count[b]);
    const int64_t slot = (int64_t)start[b] + i;
    ok = ok && slot >= 0 && slot < kv.smax;
    const int64_t row = ok ? mx_row(kv, b, h, (int)slot) : -1;
    put_block<HD, BITS>(x, kv.k, kv.k_scale, row, part);
    put_block<HD, BITS>(y, kv.v, kv.v_scale, row, part);
}

template <typename T, int HD, int BITS>
__device__ __forceinline__ void get_part(const unsigned char *codes, const uint8_t *scales, int64_t row, int part, T *dst) {
    const float scale = mx_scale(scales[row * (HD / 32) + (part >> 2)]);
    const unsigned char *src = codes + row * (HD * BITS / 8) + part * BITS;
    bf16x8 o;
    if constexpr (BITS == 4) o = mx_decode4(*reinterpret_cast<const uint32_t *>(src), scale);
    else {
        const uint2 c = *reinterpret_cast<const uint2 *>(src);
        o = mx_decode8(c.x, c.y, scale);
    }
    const uint4 u = __builtin_bit_cast(uint4, o);
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint4 *>(dst) = u;
    else {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 2; j++)
            reinterpret_cast<float4 *>(dst)[j] = make_float4(__uint_as_float(w[2 * j] << 16), __uint_as_float(w[2 * j] & 0xFFFF0000u),
                                                             __uint_as_float(w[2 * j + 1] << 16), __uint_as_float(w[2 * j + 1] & 0xFFFF0000u));
    }
}

template <typename T, int HD, int BITS>
__global__ __launch_bounds__(MX_THREADS) void kv_read_mx_kernel(KvMx kv, T *__restrict__ k, MxRows ks, T *__restrict__ v, MxRows vs, int n_slots,
                                                                const int32_t *__restrict__ start,
                                                                const int32_t *__restrict__ length) {
    constexpr int PARTS = HD / 8, ROWS = MX_THREADS / PARTS;
    const int part = threadIdx.x % PARTS, h = blockIdx.y, b = blockIdx.z;
    const int i = blockIdx.x * ROWS + threadIdx.x / PARTS;
    if (i >= min(length[b], n_slots)) return;
    const int64_t slot = (int64_t)(start ? start[b] : 0) + i;
    if (slot < 0 || slot >= kv.smax) return;
    const int64_t row = mx_row(kv, b, h, (int)slot);
    if (k) get_part<T, HD, BITS>(kv.k, kv.k_scale, row, part, k + ks.at(b, h, i) + part * 8);
    if (v) get_part<T, HD, BITS>(kv.v, kv.v_scale, row, part, v + vs.at(b, h, i) + part * 8);
}

int kv_mx_of(const bita_kv_mx *kv, KvMx *out, const char *who) {
    if (!kv->k || !kv->v || !kv->k_scale || !kv->v_scale || kv->batch <= 0 || kv->n_kv_heads <= 0 || kv->smax <= 0)
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: null cache pointer or non-positive size", who);
    if (((uintptr_t)kv->k | (uintptr_t)kv->v | (uintptr_t)kv->k_scale | (uintptr_t)kv->v_scale) & 15)
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: cache pointers must be multiples of 16 bytes", who);
    if ((kv->bits != 4 && kv->bits != 8) || (kv->head_dim != 64 && kv->head_dim != 128) || kv->n_kv_heads > 65535 || kv->batch > 65535)
        return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: bits 4 or 8, head_dim 64 or 128, at most 65535 heads and sequences", who);
    *out = KvMx{(unsigned char *)kv->k, (unsigned char *)kv->v, kv->k_scale, kv->v_scale, nullptr, kv->batch, kv->n_kv_heads, kv->smax, 0, kv->smax, -1, kv->batch, 0};
    if (!kv->block_table) return BITA_OK;
    const int ps = kv->page_size;
    if (ps < 16 || (ps & (ps - 1)) || kv->n_pages <= 0 || kv->max_pages <= 0)
        return bita_set_error(BITA_ERR_INVALID_ARG, "%s: paged cache needs page_size a power of two >= 16 (got %d), n_pages and max_pages positive", who, ps);
    if ((int64_t)kv->smax > (int64_t)kv->max_pages * ps)
        return bita_set_error(BITA_ERR_CAPACITY, "%s: smax %d exceeds the block table (%d pages of %d)", who, kv->smax, kv->max_pages, ps);
    out->table = kv->block_table;
    out->page_lg = __builtin_ctz((unsigned)ps);
    out->page_rows = ps;
    out->slot_mask = ps - 1;
    out->n_pages = kv->n_pages;
    out->max_pages = kv->max_pages;
    return BITA_OK;
}

static int check_rows(const char *who, int32_t type, int32_t n, const MxRows &ks, const MxRows &vs, const void *a, const void *b) {
    if (type != BITA_F32 && type != BITA_BF16) return bita_set_error(BITA_ERR_INVALID_ARG, "%s: type %d", who, type);
    if (n < 0 || n > MX_MAX_ROWS) return bita_set_error(BITA_ERR_INVALID_ARG, "%s: 0 to %d rows", who, MX_MAX_ROWS);
    return mx_rows_check(who, ks, vs, (uintptr_t)a | (uintptr_t)b);
}

int mx_rows_check(const char *who, const MxRows &k, const MxRows &v, uintptr_t pointers) {
    const int64_t all = k.seq | k.head | k.row | v.seq | v.head | v.row;                // (the sign bit too)
    if (all < 0) return bita_set_error(BITA_ERR_INVALID_ARG, "%s: negative stride", who);
    if (all & 7 || pointers & 15) return bita_set_error(BITA_ERR_UNSUPPORTED, "%s: strides must be multiples of 8 elements, pointers of 16 bytes", who);
    return BITA_OK;
}

#define MX_FOR(type, kv, CALL)                                                                        \
    do {                                                                                              \
        if ((type) == BITA_F32) { if ((kv)->head_dim == 128) { if ((kv)->bits == 4) CALL(float, 128, 4); else CALL(float, 128, 8); }           \
                                  else { if ((kv)->bits == 4) CALL(float, 64, 4); else CALL(float, 64, 8); } }                                 \
        else { if ((kv)->head_dim == 128) { if ((kv)->bits == 4) CALL(uint16_t, 128, 4); else CALL(uint16_t, 128, 8); }                        \
               else { if ((kv)->bits == 4) CALL(uint16_t, 64, 4); else CALL(uint16_t, 64, 8); } }                                              \
    } while (0)

extern "C" int bita_kv_write_mx(const bita_kv_mx *kv, const void *d_k, int64_t k_seq, int64_t k_head, int64_t k_row, const void *d_v, int64_t v_seq,
                                int64_t v_head, int64_t v_row, int32_t type, int32_t n_rows, const int32_t *d_start, const int32_t *d_count, const int32_t *d_path,
                                int32_t path_stride, const int32_t *d_cu_rows, void *stream) {
    if (!kv || (n_rows && (!d_k || !d_v)) || !d_start) return bita_set_error(BITA_ERR_INVALID_ARG, "bita_kv_write_mx: null argument");
    if (d_path && (d_cu_rows || path_stride <= 0 || path_stride > MX_MAX_ROWS))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_kv_write_mx: a path has a positive length and goes with rows by sequence");
    KvMx c;
    if (int rc = kv_mx_of(kv, &c, "bita_kv_write_mx")) return rc;
    const MxRows ks = mx_rows(d_cu_rows ? 1 : kv->batch, k_seq, kv->n_kv_heads, k_head, n_rows, k_row),
                 vs = mx_rows(d_cu_rows ? 1 : kv->batch, v_seq, kv->n_kv_heads, v_head, n_rows, v_row);
    if (int rc = check_rows("bita_kv_write_mx", type, n_rows, ks, vs, d_k, d_v)) return rc;
    if (n_rows == 0) return BITA_OK;
    const int per_wg = MX_THREADS * 8 / kv->head_dim;
    const int64_t wgs = (((d_path ? path_stride : n_rows) + per_wg - 1) / per_wg) * (int64_t)kv->n_kv_heads;
    if (wgs >= (1ll << 32) / MX_THREADS) return bita_set_error(BITA_ERR_UNSUPPORTED, "bita_kv_write_mx: %lld workgroups", (long long)wgs);
    const dim3 grid((unsigned)wgs, d_cu_rows ? 1 : kv->batch);
#define MX_WRITE(T_, HD_, BITS_) hipLaunchKernelGGL((kv_write_mx_kernel<T_, HD_, BITS_>), grid, dim3(MX_THREADS), 0, (hipStream_t)stream, c, (const T_ *)d_k, ks, \
                                                    (const T_ *)d_v, vs, n_rows, d_start, d_count, d_path, path_stride, d_cu_rows)
    MX_FOR(type, kv, MX_WRITE);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}

extern "C" int bita_kv_read_mx(const bita_kv_mx *kv, void *d_k, int64_t k_seq, int64_t k_head, int64_t k_row, void *d_v, int64_t v_seq, int64_t v_head,
                               int64_t v_row, int32_t out_type, int32_t n_slots, const int32_t *d_start, const int32_t *d_length, void *stream) {
    if (!kv || (n_slots && !d_k && !d_v) || !d_length) return bita_set_error(BITA_ERR_INVALID_ARG, "bita_kv_read_mx: null argument");
    KvMx c;
    if (int rc = kv_mx_of(kv, &c, "bita_kv_read_mx")) return rc;
    const MxRows ks = mx_rows(kv->batch, k_seq, kv->n_kv_heads, k_head, n_slots, k_row), vs = mx_rows(kv->batch, v_seq, kv->n_kv_heads, v_head, n_slots, v_row);
    if (int rc = check_rows("bita_kv_read_mx", out_type, n_slots, ks, vs, d_k, d_v)) return rc;
    if ((d_k && rows_overlap(kv->head_dim, {kv->batch, k_seq}, {kv->n_kv_heads, k_head}, {n_slots, k_row})) ||
        (d_v && rows_overlap(kv->head_dim, {kv->batch, v_seq}, {kv->n_kv_heads, v_head}, {n_slots, v_row})))
        return bita_set_error(BITA_ERR_INVALID_ARG, "bita_kv_read_mx: rows of an output overlap");
    if (n_slots == 0) return BITA_OK;
    const int per_wg = MX_THREADS * 8 / kv->head_dim;
    const dim3 grid((n_slots + per_wg - 1) / per_wg, kv->n_kv_heads, kv->batch);
#define MX_READ(T_, HD_, BITS_) hipLaunchKernelGGL((kv_read_mx_kernel<T_, HD_, BITS_>), grid, dim3(MX_THREADS), 0, (hipStream_t)stream, c, (T_ *)d_k, ks, (T_ *)d_v, \
                                                   vs, n_slots, d_start, d_length)
    MX_FOR(out_type, kv, MX_READ);
    BITA_HIP_CHECK(hipGetLastError());
    return BITA_OK;
}
