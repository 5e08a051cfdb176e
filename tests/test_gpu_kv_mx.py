"""The 4- and 8-bit K/V cache: rows rounded as they are written, and read back (GPU)."""
import pytest
import torch

import mx_reference as ref

pytestmark = pytest.mark.gpu
BITS = pytest.mark.parametrize("bits", [4, 8])


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def make(hkv, hd, n, smax, bits, page=0, seed=0):
    import paper_2401_12522_amd as bita
    table = None
    if page:
        per = -(-smax // page)
        table = torch.randperm(n * per + 3, generator=torch.Generator().manual_seed(seed))[: n * per].to(torch.int32).view(n, per).cuda()
        return bita.KVCacheMX(hkv, hd, n, smax, bits=bits, block_table=table, page_size=page, n_pages=n * per + 3)
    return bita.KVCacheMX(hkv, hd, n, smax, bits=bits)


def slots(cache, t):
    """A cache tensor as [n][hkv][smax][w] on the CPU."""
    t = t.cpu()
    if cache.block_table is None:
        return t
    return t[cache.block_table.long().cpu()].transpose(1, 2).flatten(2, 3)[:, :, : cache.smax]


def rows(shape, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(torch.randn(shape[:-1], generator=g))[..., None]
    return x.to(dtype)


def check(cache, k, v, n, start, count=None):
    """Slots start .. of every sequence hold the blocks of k, v [n][hkv][rows][hd]; all others are as they were made."""
    for codes, scales, x in ((cache.k, cache.k_scale, k), (cache.v, cache.v_scale, v)):
        codes, scales = slots(cache, codes), slots(cache, scales)
        want_c = torch.zeros_like(codes)
        want_s = torch.full_like(scales, 127)
        c, s = ref.quantize(x, cache.bits)
        c = ref.pack(c, cache.bits)
        for b in range(n):
            for i in range(x.shape[2] if count is None else min(count[b], x.shape[2])):
                if 0 <= start[b] + i < cache.smax:
                    want_c[b, :, start[b] + i], want_s[b, :, start[b] + i] = c[b, :, i], s[b, :, i]
        assert torch.equal(scales, want_s)
        assert torch.equal(codes, want_c)


@BITS
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd,page", [(128, 0), (64, 16), (128, 64), (64, 0)])
def test_rows_of_sequences(bits, dtype, hd, page):
    import paper_2401_12522_amd as bita
    n, hkv, m = 3, 2, 21
    cache = make(hkv, hd, n, 60, bits, page)
    k, v = rows((n, hkv, m, hd), 1, dtype), rows((n, hkv, m, hd), 2, dtype)
    start, count = [0, 39, 50], [21, 0, 21]                      # the last one's rows pass the end: dropped
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), i32(start), i32(count))
    check(cache, k, v, n, start, count)


@BITS
def test_every_exponent_tie_and_border(bits):
    """Blocks of every size from subnormal to the largest numbers; in each, values at and next to the borders between codes."""
    import paper_2401_12522_amd as bita
    g = ref.grid(bits)
    mids = (g[1:] + g[:-1]) / 2
    some = torch.cat([g, mids])[torch.randperm(len(g) * 2 - 1, generator=torch.Generator().manual_seed(3))[:10]]
    out = []
    for e in range(-149, 128):
        for top in (1.0, 1.7499, 1.75, 1.8125, 1.8126, 1.9999):
            scale = top * 2.0 ** (e if e < 127 else 127)
            unit = 2.0 ** (e - (2 if bits == 4 else 8))          # near the block's 2^e
            near = torch.cat([some * unit, torch.nextafter((some * unit).float(), torch.tensor(0.0)).double(),
                              torch.nextafter((some * unit).float(), torch.tensor(3e38)).double()])
            near = torch.where(near.abs() <= scale, near, torch.zeros(()).double())
            out.append(torch.cat([torch.tensor([scale], dtype=torch.float64), near, torch.zeros(1).double()]) * torch.tensor([1, -1]).repeat(16))
    x = torch.stack(out).float()
    x = torch.cat([x, torch.zeros((-len(x)) % 4, 32)]).view(1, 1, -1, 128)
    cache = make(1, 128, 1, x.shape[2], bits)
    bita.kv_write_mx(cache, x.cuda(), (-x).cuda(), i32([0]))
    check(cache, x, -x, 1, [0])


@BITS
def test_infinities_nan_and_zeros(bits):
    import paper_2401_12522_amd as bita
    x = rows((1, 1, 6, 128), 4)
    x[0, 0, 0, 5], x[0, 0, 1, 40], x[0, 0, 2, 127], x[0, 0, 3] = float("nan"), float("inf"), float("-inf"), 0.0
    cache = make(1, 128, 1, 6, bits)
    bita.kv_write_mx(cache, x.cuda(), x.cuda(), i32([0]))
    check(cache, x, x, 1, [0])
    for dtype in (torch.bfloat16, torch.float32):
        k, v = (torch.empty((1, 1, 6, 128), dtype=dtype, device="cuda") for _ in range(2))
        bita.kv_read_mx(cache, k, v, i32([6]))
        want = ref.rounded(x, bits)
        assert torch.equal(k.cpu().double().nan_to_num(1e30), want.nan_to_num(1e30))
        assert torch.equal(v.cpu().double().nan_to_num(1e30), want.nan_to_num(1e30))


@BITS
def test_every_code_reads_back(bits):
    """All codes with every scale byte that is written (and 255)."""
    import paper_2401_12522_amd as bita
    lo = ref.LOWEST[bits] + 127
    scale = torch.tensor(list(range(lo, 253 if bits == 4 else 247)) + [255], dtype=torch.uint8)
    code = torch.arange(256 if bits == 8 else 16)
    code = code[(code & 127) != 127] if bits == 8 else code     # (the 8-bit NaN codes are never written)
    n = -(-len(code) // 32) * 32
    code = torch.cat([code, code[: n - len(code)]]).to(torch.uint8)
    pairs = [(code[i: i + 32], s) for s in scale for i in range(0, n, 32)]
    pairs += pairs[: (-len(pairs)) % 2]
    c = torch.stack([p[0] for p in pairs]).view(1, 1, -1, 64)
    s = torch.stack([p[1] for p in pairs]).view(1, 1, -1, 2)
    cache = bita.KVCacheMX(1, 64, 1, c.shape[2], bits=bits, k=ref.pack(c, bits).contiguous().cuda(), v=ref.pack(c, bits).contiguous().cuda(), k_scale=s.cuda(), v_scale=s.cuda())
    want = ref.values(c, s, bits).nan_to_num(1e39)
    for dtype in (torch.bfloat16, torch.float32):
        k = torch.empty((1, 1, c.shape[2], 64), dtype=dtype, device="cuda")
        bita.kv_read_mx(cache, k, None, i32([c.shape[2]]))
        assert torch.equal(k.cpu().double().nan_to_num(1e39), want)


@BITS
@pytest.mark.parametrize("hd,page,dtype", [(128, 0, torch.bfloat16), (64, 32, torch.float32)])
def test_packed_rows(bits, hd, page, dtype):
    """Prompts one behind the other (empty ones, single rows, rows behind the last, more than 64 of them), columns of a wider tensor."""
    import paper_2401_12522_amd as bita
    lens = [7, 0, 0, 1, 33, 0, 2] + [i % 3 for i in range(130)] + [0]
    n, hkv = len(lens), 3
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    wide = rows((cu[-1] + 5, 2 * hkv, hd), 6, dtype)
    cache = make(hkv, hd, n, 40, bits, page)
    start = [i % 4 for i in range(n)]
    w = wide.cuda()
    bita.kv_write_mx(cache, w[:, :hkv], w[:, hkv:], i32(start), cu_rows=i32(cu))
    k, v = torch.zeros(2, n, hkv, 33, hd)
    for b in range(n):
        k[b, :, : lens[b]] = wide[cu[b]: cu[b + 1], :hkv].transpose(0, 1).float()
        v[b, :, : lens[b]] = wide[cu[b]: cu[b + 1], hkv:].transpose(0, 1).float()
    check(cache, k, v, n, start, lens)


@pytest.mark.parametrize("n", [1, 63, 64, 65, 4097, 5000])
def test_packed_rows_of_very_many_sequences(n):
    import paper_2401_12522_amd as bita
    lens = [(i * 5) % 3 for i in range(n)]
    cu = [3]                                                     # (rows before the first sequence are nobody's)
    for x in lens:
        cu.append(cu[-1] + x)
    k = rows((cu[-1] + 2, 1, 64), n)
    cache = make(1, 64, n, 3, 4)
    bita.kv_write_mx(cache, k.cuda(), k.cuda(), i32([0] * n), cu_rows=i32(cu))
    c, s = ref.quantize(k, 4)
    c = ref.pack(c, 4)
    want_c, want_s = torch.zeros(n, 3, 32, dtype=torch.uint8), torch.full((n, 3, 2), 127, dtype=torch.uint8)
    for b in range(n):
        want_c[b, : lens[b]], want_s[b, : lens[b]] = c[cu[b]: cu[b + 1], 0], s[cu[b]: cu[b + 1], 0]
    assert torch.equal(cache.k.cpu()[:, 0], want_c) and torch.equal(cache.v_scale.cpu()[:, 0], want_s)


@BITS
def test_accepted_rows_by_their_path(bits):
    import paper_2401_12522_amd as bita
    n, hkv, hd = 3, 2, 64
    k, v = rows((n, hkv, 9, hd), 7, torch.bfloat16), rows((n, hkv, 9, hd), 8, torch.bfloat16)
    path = [[0, 4, 8, -1], [0, -1, -1, -1], [0, 3, 3, 100]]     # padding is not written; a row past the pass is clamped
    acc, start = [3, 1, 4], [5, 0, 17]
    cache = make(hkv, hd, n, 21, bits)
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), i32(start), i32(acc), path=i32(path))
    pick = torch.tensor(path).clamp(0, 8)
    take = lambda t: torch.stack([t[b][:, pick[b]] for b in range(n)])           # noqa: E731
    check(cache, take(k), take(v), n, start, acc)


@BITS
@pytest.mark.parametrize("page", [0, 16])
def test_parts_read_back_and_nothing_else_written(bits, page):
    import paper_2401_12522_amd as bita
    n, hkv, hd, smax = 3, 2, 128, 50
    cache = make(hkv, hd, n, smax, bits, page)
    k, v = rows((n, hkv, smax, hd), 9), rows((n, hkv, smax, hd), 10)
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), i32([0] * n))
    first, length = [0, 13, 45], [17, -3, 9]                    # a negative length, a length past the cache
    out = torch.full((n, 20, 2 * hkv, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    bita.kv_read_mx(cache, out[:, :, :hkv].transpose(1, 2), out[:, :, hkv:].transpose(1, 2), i32(length), start=i32(first))
    want = torch.full((n, 20, 2 * hkv, hd), 7.0, dtype=torch.float64)
    rk, rv = ref.rounded(k, bits), ref.rounded(v, bits)
    for b in range(n):
        for i in range(min(max(length[b], 0), 20)):
            if first[b] + i < smax:
                want[b, i, :hkv], want[b, i, hkv:] = rk[b, :, first[b] + i], rv[b, :, first[b] + i]
    assert torch.equal(out.cpu().double(), want)


def test_error_of_a_block_is_half_a_step_of_its_largest_binade():
    """|v - read back| <= 2^e: half the spacing of the largest codes (2 2^e in 4 bits, 32 2^e in 8)."""
    import paper_2401_12522_amd as bita
    x = rows((1, 4, 300, 128), 11)
    for bits, half in ((4, 1.0), (8, 16.0)):
        cache = make(4, 128, 1, 300, bits)
        bita.kv_write_mx(cache, x.cuda(), x.cuda(), i32([0]))
        k = torch.empty_like(x, device="cuda")
        bita.kv_read_mx(cache, k, None, i32([300]))
        step = 2.0 ** (slots(cache, cache.k_scale).double() - 127) * half
        assert ((k.cpu() - x).double().abs() <= step.repeat_interleave(32, -1)).all()


def test_bad_pages_and_starts_stay_in_the_pool():
    """Page ids outside the pool are clamped; starts outside the cache write nothing."""
    import paper_2401_12522_amd as bita
    table = i32([[-5, 1000], [2, 1]])
    cache = bita.KVCacheMX(1, 64, 2, 32, bits=4, block_table=table, page_size=16, n_pages=4)
    k = rows((2, 1, 40, 64), 12).cuda()
    bita.kv_write_mx(cache, k, k, i32([0, -2 ** 31]))
    c, s = ref.quantize(k.cpu(), 4)
    c = ref.pack(c, 4)
    assert torch.equal(cache.k.cpu()[0, 0], c[0, 0, :16]) and torch.equal(cache.k.cpu()[3, 0], c[0, 0, 16:32])
    assert not cache.k[1:3].any()
    bita.kv_write_mx(cache, k, k, i32([2 ** 31 - 1, 31]))
    assert not cache.k[2].any() and torch.equal(cache.k.cpu()[1, 0, 15], c[1, 0, 0]) and not cache.k[1, 0, :15].any()


def test_far_slots():
    """Offsets of a cache beyond 2^32 bytes, and beyond 2^31 elements of what is read back."""
    import paper_2401_12522_amd as bita
    hkv, hd, smax = 8, 128, 4_300_000
    cache = bita.KVCacheMX(hkv, hd, 2, smax, bits=8)
    assert cache.k.numel() > 2 ** 32
    k, v = rows((2, hkv, 5, hd), 13, torch.bfloat16), rows((2, hkv, 5, hd), 14, torch.bfloat16)
    at = i32([smax - 5, smax - 7])
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), at)
    assert torch.equal(cache.k[1, 7, smax - 7: smax - 2].cpu(), ref.quantize(k[1, 7], 8)[0])
    out = torch.empty((2, hkv, 5, hd), dtype=torch.bfloat16, device="cuda")
    bita.kv_read_mx(cache, out, None, i32([5, 5]), start=at)
    assert torch.equal(out.cpu().double(), ref.rounded(k, 8))
