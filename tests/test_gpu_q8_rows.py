"""Rows as 8-bit integers (GPU): norm, gating and plain rows against their definition in 64 bits.  Every integer has to be the
definition's; a scale is off by its one rounding to 32 bits (half a step, 2^-24 of it)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def definition(v):
    """(q, s) of rows of doubles."""
    top = v.abs().max(1, keepdim=True).values
    t = v.abs() * 127 / torch.where(top > 0, top, 1.0)
    low = torch.floor(t)
    up = (t - low > 0.5) | ((t - low == 0.5) & (low % 2 == 1))
    return ((low + up) * torch.sign(v)).to(torch.int8), top[:, 0] / 127


def check(q, scale, v, factor=None):
    want, s = definition(v)
    s = s if factor is None else s * factor
    assert torch.equal(q, want), f"{int((q != want).sum())} of {q.numel()} integers differ"
    assert bool(((scale.double() - s).abs() <= 2.0 ** -24 * 1.0001 * s + 2.0 ** -149).all())


def rows(m, k, seed, dtype, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(m, k, device="cuda", generator=g) * torch.exp(spread * torch.randn(k, device="cuda", generator=g))).to(dtype)


SIZES = [(1, 1), (1, 7), (3, 8), (2, 63), (5, 64), (1, 513), (4, 1000), (68, 4096), (1, 5115), (3, 8191), (2, 8192), (2, 8193), (3, 16384), (2, 16385),
         (1, 28672), (2, 32768), (2, 32769), (1, 70001), (1, 131071), (700, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k", SIZES)
def test_plain_rows(m, k, dtype):
    import paper_2401_12522_amd as bita
    x = rows(m, k, m + k, TYPES[dtype])
    check(*bita.quantize_rows(x), x.double())


@pytest.mark.parametrize("x_type,delta_type", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", None), ("bf16", None)])
@pytest.mark.parametrize("m,d", [s for s in SIZES if s[1] <= 16384])
def test_norm(m, d, x_type, delta_type):
    import paper_2401_12522_amd as bita
    x, eps = rows(m, d, m + d, TYPES[x_type]), 1e-5
    gain = rows(1, d, 3, torch.bfloat16, 0.1)[0]
    h, delta, total = x.clone(), None, None
    if delta_type:
        delta = rows(m, d, 7, TYPES[delta_type])
        h = (x.float() + delta.float()).to(x.dtype)
        total = torch.empty_like(x)
    before = x.clone()
    q, scale = bita.norm_q8(x, gain, eps, delta=delta, total=total)
    assert torch.equal(x, before)
    if total is not None:
        assert torch.equal(total, h)
    r = 1 / torch.sqrt(h.double().square().mean(1) + eps)
    check(q, scale, h.double() * gain.double(), r)
    if delta is not None:                                            # in place
        q2, scale2 = bita.norm_q8(x, gain, eps, delta=delta)
        assert torch.equal(x, h) and torch.equal(q2, q) and torch.equal(scale2, scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tile", [0, 16])
@pytest.mark.parametrize("m,f", SIZES)
def test_gating(m, f, tile, dtype):
    import paper_2401_12522_amd as bita
    f = min((f + 15) // 16 * 16, 131056) if tile else f             # (131071 columns at most, whole tiles)
    x = rows(m, 2 * f, m + f, TYPES[dtype])
    gate, up = (x.view(m, f // 16, 2, 16).unbind(2) if tile else (x[:, :f], x[:, f:]))
    gate, up = gate.reshape(m, f).double(), up.reshape(m, f).double()
    check(*bita.silu_mul_q8(x, tile=tile), gate / (1 + torch.exp(-gate)) * up)


@pytest.mark.parametrize("top", [127.0, 254.0, 63.5, 127.0 * 2 ** -40, 127.0 * 2 ** 60])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_go_to_even(dtype, top):
    """Rows of half steps: every other value lies on a border."""
    import paper_2401_12522_amd as bita
    half = torch.arange(-254, 255, device="cuda", dtype=torch.float64) * (top / 254)
    x = half.to(TYPES[dtype])
    x = x[x.double() == half][None].contiguous()                    # (bf16: those it holds)
    assert x.shape[1] > 250 and float(x.abs().max()) == top
    check(*bita.quantize_rows(x), x.double())
    gain = torch.ones(x.shape[1], dtype=torch.bfloat16, device="cuda")
    check(*bita.norm_q8(x, gain, 0.0), x.double(), 1 / x.double().square().mean(1).sqrt())


def test_values_next_to_a_border():
    """fp32 neighbours of the borders, where a quotient in fp32 lands on the border itself."""
    import paper_2401_12522_amd as bita
    g = torch.Generator(device="cuda").manual_seed(5)
    top = torch.rand(64, 1, device="cuda", generator=g, dtype=torch.float64).float() + 1
    k = torch.randint(0, 127, (64, 2000), device="cuda", generator=g)
    x = ((k + 0.5) * top.double() / 127).float()
    step = torch.randint(-2, 3, x.shape, device="cuda", generator=g, dtype=torch.int32)
    x = (x.view(torch.int32) + step).view(torch.float32)
    x[:, 0] = top[:, 0]
    check(*bita.quantize_rows(x), x.double())
    gate = torch.full_like(x, 20.0)                                  # silu(20) = 20 / (1 + e^-20)
    pair = torch.cat([gate, x], 1)
    check(*bita.silu_mul_q8(pair), 20 / (1 + torch.exp(torch.tensor(-20.0, dtype=torch.float64, device="cuda"))) * x.double())


@pytest.mark.parametrize("size", [1e-42, 1e-37, 1e-20, 1e20, 3e37])
def test_values_at_the_ends_of_the_range(size):
    import paper_2401_12522_amd as bita
    x = (rows(3, 1000, 1, torch.float32, 0.3).clamp(-4, 4) * size).contiguous()
    check(*bita.quantize_rows(x), x.double())
    gain = rows(1, 1000, 2, torch.bfloat16, 0.1)[0]
    check(*bita.norm_q8(x, gain, 0.0), x.double() * gain.double(), 1 / x.double().square().mean(1).sqrt())
    if size < 1:
        gate = rows(3, 1000, 4, torch.float32, 0.1)
        check(*bita.silu_mul_q8(torch.cat([gate, x], 1)), gate.double() / (1 + torch.exp(-gate.double())) * x.double())


def test_gates_far_below_zero():
    """exp(-gate) beyond fp32: the whole row is tiny, and still rounded by its own largest value."""
    import paper_2401_12522_amd as bita
    gate = -85 - 20 * torch.rand(2, 300, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    up = rows(2, 300, 2, torch.float32, 0.2)
    v = gate.double() / (1 + torch.exp(-gate.double())) * up.double()
    check(*bita.silu_mul_q8(torch.cat([gate, up], 1)), v)


@pytest.mark.parametrize("call", ["rows", "norm", "gate"])
def test_rows_of_zeros_and_of_no_number(call):
    import paper_2401_12522_amd as bita
    k = 500
    x = rows(6, 2 * k if call == "gate" else k, 1, torch.float32)
    x[1] = 0
    x[2, 77] = float("nan")
    x[3, 3] = float("inf")
    x[4, k - 1] = float("-inf")
    x[5, :] = float("inf")
    if call == "gate":
        x[:, k + 77] = 1.0
        x[4, 2 * k - 1] = 2.0
        x[4, k - 1] = float("inf")
        q, scale = bita.silu_mul_q8(x)
        want = x[:1, :k].double() / (1 + torch.exp(-x[:1, :k].double())) * x[:1, k:].double()
    elif call == "norm":
        gain = torch.ones(k, dtype=torch.bfloat16, device="cuda")
        q, scale = bita.norm_q8(x, gain, 0.0)
        want = x[:1].double()
    else:
        q, scale = bita.quantize_rows(x)
        want = x[:1].double()
    assert torch.equal(q[:1], definition(want)[0])
    assert not q[1:].any()
    assert float(scale[0]) > 0 and float(scale[1]) == 0 and bool(torch.isnan(scale[2:]).all())


def test_strides_offsets_and_what_lies_around_the_rows():
    """Rows inside larger tensors, at odd offsets: the same numbers, and nothing else is written."""
    import paper_2401_12522_amd as bita
    m, k = 5, 1003
    for dtype in (torch.float32, torch.bfloat16):
        for off, ld in ((0, 1040), (1, 1041), (8, 1048), (3, 1056)):
            big = rows(m + 2, ld, 1, dtype)
            x = big[1:-1, off:off + k]
            qbig = torch.full((m + 2, ld), 99, dtype=torch.int8, device="cuda")
            sbig = torch.full((m + 2,), -1.0, device="cuda")
            q, scale = bita.quantize_rows(x, q=qbig[1:-1, off:off + k], scale=sbig[1:-1])
            check(q, scale, x.double())
            qbig[1:-1, off:off + k] = 99
            assert bool((qbig == 99).all()) and float(sbig[0]) == float(sbig[-1]) == -1
            gain = rows(1, k + 1, 2, torch.bfloat16, 0.1)[0, off % 2: off % 2 + k]
            tbig = torch.full((m + 2, ld), 5.0, dtype=dtype, device="cuda")
            delta = rows(m, ld + 1, 3, torch.float32)[:, 1:k + 1]
            q, scale = bita.norm_q8(x, gain.contiguous(), 1e-5, delta=delta, total=tbig[1:-1, off:off + k], q=qbig[1:-1, off:off + k], scale=sbig[1:-1])
            h = (x.float() + delta).to(dtype)
            assert torch.equal(tbig[1:-1, off:off + k], h)
            check(q, scale, h.double() * gain.double(), 1 / torch.sqrt(h.double().square().mean(1) + 1e-5))
            tbig[1:-1, off:off + k] = 5.0
            qbig[1:-1, off:off + k] = 99
            assert bool((qbig == 99).all()) and bool((tbig == 5.0).all())
            f = k // 2
            q, scale = bita.silu_mul_q8(x[:, :2 * f], q=qbig[1:-1, off:off + f], scale=sbig[1:-1])
            gate, up = x[:, :f].double(), x[:, f:2 * f].double()
            check(q, scale, gate / (1 + torch.exp(-gate)) * up)
            qbig[1:-1, off:off + f] = 99
            assert bool((qbig == 99).all()) and float(sbig[0]) == float(sbig[-1]) == -1


@pytest.mark.parametrize("call", ["rows", "norm", "gate"])
def test_more_rows_than_a_launch_has(call):
    import paper_2401_12522_amd as bita
    m, k = (1 << 21) + 5, 9
    x = rows(m, 2 * k if call == "gate" else k, 5, torch.bfloat16)
    if call == "rows":
        q, s = bita.quantize_rows(x)
        v, factor = x.double(), None
    elif call == "norm":
        delta, total, gain = rows(m, k, 6, torch.float32), torch.empty_like(x), rows(1, k, 7, torch.bfloat16, 0.1)[0]
        q, s = bita.norm_q8(x, gain, 1e-5, delta=delta, total=total)
        h = (x.float() + delta).bfloat16()
        assert torch.equal(total, h)
        v, factor = h.double() * gain.double(), 1 / torch.sqrt(h.double().square().mean(1) + 1e-5)
    else:
        q, s = bita.silu_mul_q8(x)
        g, u = x[:, :k].double(), x[:, k:].double()
        v, factor = g / (1 + torch.exp(-g)) * u, None
    check(q, s, v, factor)


def test_refusals_of_the_binding():
    import paper_2401_12522_amd as bita
    x = rows(4, 64, 1, torch.float32)
    gain = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: bita.quantize_rows(x.half()), lambda: bita.quantize_rows(x.T), lambda: bita.quantize_rows(x[0]), lambda: bita.quantize_rows(x.cpu()),
                lambda: bita.quantize_rows(x[:0]), lambda: bita.quantize_rows(x[:1].expand(4, 64)), lambda: bita.quantize_rows(x, q=bita.empty_q8(4, 63)),
                lambda: bita.quantize_rows(x, scale=torch.empty(3, device="cuda")), lambda: bita.norm_q8(x, gain[:63], 1e-5),
                lambda: bita.norm_q8(x, gain.float(), 1e-5), lambda: bita.norm_q8(x, gain, 1e-5, delta=x[:3]),
                lambda: bita.norm_q8(x, gain, 1e-5, total=x), lambda: bita.norm_q8(x, gain, 1e-5, delta=x, total=x.to(torch.bfloat16)),
                lambda: bita.silu_mul_q8(x[:, :63])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(bita.BitaError):
        bita.silu_mul_q8(x, tile=8)
