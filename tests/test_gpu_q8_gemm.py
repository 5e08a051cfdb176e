"""The product of 8-bit integers with scales (GPU), against sums in 64-bit integers.  The sums are exact; an fp32 output has
three roundings of half a step (the sum to fp32, two products): 3 * 2^-24 and their products; a bf16 output one of 2^-8 more."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BOUND = {torch.float32: 3.01 * 2.0 ** -24, torch.bfloat16: 2.0 ** -8 + 4 * 2.0 ** -24}


def codes(m, k, seed, lo=-127, hi=128):
    g = torch.Generator(device="cuda").manual_seed(seed)
    import paper_2401_12522_amd as bita
    q = bita.empty_q8(m, k)
    q.copy_(torch.randint(lo, hi, (m, k), device="cuda", generator=g))
    return q, torch.rand(m, device="cuda", generator=g) * 0.01 + 0.001


def exact_sums(a, w):
    """Whole sums: doubles hold them."""
    return a.double() @ w.double().T


def check(y, a, sa, w, sw):
    want = exact_sums(a, w) * sa.double()[:, None] * sw.double()
    off = (y.double() - want).abs()
    assert y.shape == want.shape
    worst = float((off - BOUND[y.dtype] * want.abs()).max())
    assert worst <= 0, f"{int((off > BOUND[y.dtype] * want.abs()).sum())} of {y.numel()} off, first at {(off > BOUND[y.dtype] * want.abs()).nonzero()[0].tolist()}"


SIZES = [(1, 1, 1), (1, 16, 64), (2, 17, 129), (16, 64, 128), (5, 100, 1000), (1, 4096, 4096), (17, 1037, 2731), (33, 48, 16), (48, 4096, 512),
         (64, 200, 11008), (65, 12288, 257), (68, 22016, 4096), (80, 8192, 1024), (81, 500, 640), (96, 4096, 4096), (100, 3000, 3001), (128, 256, 384), (129, 1000, 130),
         (160, 2049, 512), (171, 12288, 96), (256, 512, 256), (272, 4096, 1376), (300, 1111, 5115), (512, 2048, 1024), (513, 777, 200), (1000, 130, 1000),
         (1024, 4096, 640), (2111, 300, 77), (4096, 32, 128)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product(m, n, k, dtype):
    import paper_2401_12522_amd as bita
    (a, sa), (w, sw) = codes(m, k, 1), codes(n, k, 2)
    out = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
    y = bita.gemm_q8(a, sa, bita.pack_weight_q8(w), sw, n, out=out)
    assert y is out
    check(y, a, sa, w, sw)


@pytest.mark.parametrize("m,n,k,rows,cols,splits", [
    # every workgroup shape, k whole and split, ragged at every end
    (3, 64, 28672, 16, 16, 8), (16, 200, 9000, 16, 16, 4), (1, 4165, 107515, 16, 32, 1), (39, 8303, 10455, 48, 128, 3), (34, 3166, 21811, 48, 64, 5), (50, 28702, 2, 64, 128, 1),
    (68, 1037, 11000, 80, 32, 5), (83, 3006, 23350, 96, 96, 8), (86, 916, 119981, 96, 32, 8), (109, 32758, 374, 112, 128, 1), (117, 1504, 61018, 128, 48, 8), (144, 22016, 300, 144, 128, 1),
    (275, 4021, 189, 144, 32, 1), (160, 48, 131071, 80, 16, 8), (79, 79711, 905, 96, 192, 1), (144, 500, 9001, 144, 16, 4), (700, 300, 20000, 128, 128, 8),
    (300, 100, 131071, 128, 128, 8), (1500, 130, 4001, 128, 128, 4), (149, 34781, 21400, 160, 256, 3), (293, 32003, 400, 160, 256, 1), (520, 9000, 400, 128, 256, 1),
    (898, 12646, 1507, 256, 256, 1), (33, 8313, 16, 48, 48, 1), (135, 5457, 7824, 144, 128, 4), (281, 22543, 16, 288, 128, 1), (281, 22543, 515, 288, 128, 1),
    (4244, 283, 5726, 288, 128, 5)])
def test_workgroup_shapes(m, n, k, rows, cols, splits):
    import paper_2401_12522_amd as bita
    plan = bita.binding.gemm_q8_plan_info(m, n, k)
    assert (plan["rows"], plan["cols"], plan["splits"]) == (rows, cols, splits), plan
    (a, sa), (w, sw) = codes(m, k, 1), codes(n, k, 2)
    need = bita.lib().bita_gemm_q8_workspace_bytes(m, n, k)
    assert need == (splits * m * ((n + 15) // 16 * 16) * 4 if splits > 1 else 0)
    packed, ws = bita.pack_weight_q8(w), torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
        bita.gemm_q8(a, sa, packed, sw, n, out=out, workspace=ws)
        check(out, a, sa, w, sw)
    assert bool((ws[need:] == 0xA5).all())


def test_longest_sums():
    """The largest sums there are: all -128 over the longest k."""
    import paper_2401_12522_amd as bita
    k = 131071
    a, w = bita.empty_q8(3, k), bita.empty_q8(20, k)
    a.fill_(-128)
    w.fill_(-128)
    w[1] = 127
    w[2, ::2] = 127
    one = torch.ones(20, device="cuda")
    y = bita.gemm_q8(a, one[:3].contiguous(), bita.pack_weight_q8(w), one, 20)
    check(y, a, one[:3], w, one)


def test_integers_come_out_whole():
    """Sums below 2^24 with scales of one are the sums."""
    import paper_2401_12522_amd as bita
    (a, _), (w, _) = codes(70, 1000, 3), codes(150, 1000, 4)
    y = bita.gemm_q8(a, torch.ones(70, device="cuda"), bita.pack_weight_q8(w), torch.ones(150, device="cuda"), 150)
    assert torch.equal(y.double(), exact_sums(a, w))


def test_whatever_lies_behind_a_row():
    """Columns behind k are read and multiplied with nothing; so is the weight's padding."""
    import paper_2401_12522_amd as bita
    for m, n, k in ((3, 50, 1001), (90, 300, 700), (300, 600, 1601)):
        (a, sa), (w, sw) = codes(m, k, 5), codes(n, k, 6)
        wide = torch.full((m, (k + 15) // 16 * 16 + 64), 113, dtype=torch.int8, device="cuda")
        wide[:, :k] = a
        y = bita.gemm_q8(wide[:, :k], sa, bita.pack_weight_q8(w), sw, n)
        check(y, a, sa, w, sw)


def test_rows_with_no_number_and_of_zeros():
    import paper_2401_12522_amd as bita
    for m in (4, 130, 300):
        (a, sa), (w, sw) = codes(m, 256, 5), codes(96, 256, 6)
        a[1], sa[1] = 0, float("nan")
        a[2], sa[2] = 0, 0.0
        for dtype in (torch.float32, torch.bfloat16):
            y = bita.gemm_q8(a, sa, bita.pack_weight_q8(w), sw, 96, out_dtype=dtype)
            assert bool(torch.isnan(y[1]).all()) and not y[2].any() and bool(torch.isfinite(y[3:]).all())


def test_an_output_inside_a_larger_one():
    import paper_2401_12522_amd as bita
    for m, n, k in ((5, 37, 200), (100, 200, 128), (257, 301, 300)):
        (a, sa), (w, sw) = codes(m, k, 7), codes(n, k, 8)
        for dtype in (torch.float32, torch.bfloat16):
            big = torch.full((m + 2, n + 11), 7.0, dtype=dtype, device="cuda")
            bita.gemm_q8(a, sa, bita.pack_weight_q8(w), sw, n, out=big[1:-1, 3:n + 3])
            check(big[1:-1, 3:n + 3], a, sa, w, sw)
            big[1:-1, 3:n + 3] = 7.0
            assert bool((big == 7.0).all())


def test_packing_into_a_shared_buffer():
    """Two matrices side by side and interleaved by tiles, as the gate and up weights of a layer are."""
    import paper_2401_12522_amd as bita
    (a, sa), (w1, s1), (w2, s2) = codes(70, 300, 1), codes(64, 300, 2), codes(64, 300, 3)
    both = torch.empty(bita.packed_q8_bytes(128, 300), dtype=torch.uint8, device="cuda")
    bita.pack_weight_q8(w1, both, 0, 2, total_rows=128)
    bita.pack_weight_q8(w2, both, 1, 2, total_rows=128)
    order = torch.stack([w1.view(4, 16, 300), w2.view(4, 16, 300)], 1).reshape(128, 300)
    scales = torch.stack([s1.view(4, 16), s2.view(4, 16)], 1).reshape(128)
    assert torch.equal(both, bita.pack_weight_q8(order))
    check(bita.gemm_q8(a, sa, both, scales, 128), a, sa, order, scales)
    ragged = torch.empty(bita.packed_q8_bytes(114, 300), dtype=torch.uint8, device="cuda")
    bita.pack_weight_q8(w1, ragged, 0, 1, total_rows=114)
    bita.pack_weight_q8(w2[:50], ragged, 4, 1, total_rows=114)
    scales = torch.cat([s1, s2[:50]])
    check(bita.gemm_q8(a, sa, ragged, scales, 114), a, sa, torch.cat([w1, w2[:50]]), scales)


def test_packing_from_any_alignment():
    import paper_2401_12522_amd as bita
    for off in (0, 1, 3, 16):
        big = torch.randint(-127, 128, (40, 333), device="cuda", dtype=torch.int8, generator=torch.Generator(device="cuda").manual_seed(off))
        w = big[:, off:off + 301]
        (a, sa), sw = codes(9, 301, 1), torch.ones(40, device="cuda")
        check(bita.gemm_q8(a, sa, bita.pack_weight_q8(w), sw, 40), a, sa, w, sw)


def test_the_same_call_twice_and_on_another_stream():
    import paper_2401_12522_amd as bita
    for m, n, k in ((5, 4096, 1000), (100, 1000, 4096), (700, 2000, 512)):
        (a, sa), (w, sw) = codes(m, k, 7), codes(n, k, 8)
        packed = bita.pack_weight_q8(w)
        y = bita.gemm_q8(a, sa, packed, sw, n)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            z = bita.gemm_q8(a, sa, packed, sw, n)
        side.synchronize()
        assert torch.equal(y, z)


def test_refusals_of_the_binding():
    import paper_2401_12522_amd as bita
    (a, sa), (w, sw) = codes(4, 64, 1), codes(32, 64, 2)
    packed = bita.pack_weight_q8(w)
    odd = torch.zeros((4, 72), dtype=torch.int8, device="cuda")
    tight = torch.zeros(4 * 64 - 8, dtype=torch.int8, device="cuda").as_strided((4, 56), (64, 1))
    for bad in (lambda: bita.gemm_q8(a.float(), sa, packed, sw, 32), lambda: bita.gemm_q8(a, sa[:3], packed, sw, 32), lambda: bita.gemm_q8(a, sa, packed[:-1], sw, 32),
                lambda: bita.gemm_q8(a, sa, packed, sw, 33), lambda: bita.gemm_q8(a, sa, packed, sw, 32, out=torch.empty(4, 31, device="cuda")),
                lambda: bita.gemm_q8(a, sa, packed, sw, 32, out=torch.empty(4, 32, device="cuda", dtype=torch.float16)),
                lambda: bita.gemm_q8(odd, sa, packed, sw, 32), lambda: bita.gemm_q8(odd[:, 8:], sa, packed, sw, 32), lambda: bita.gemm_q8(tight, sa, packed, sw, 32),
                lambda: bita.pack_weight_q8(w.float()), lambda: bita.pack_weight_q8(w, dst=packed[:-1])):
        with pytest.raises(ValueError):
            bad()
