"""Gating at the ends of the gates' range (GPU): gates whose exponent passes fp32 and subnormal ones, against silu(g) u in 64 bits.  Every integer has to be
the definition's, a scale within its one rounding to 32 bits."""
import pytest
import torch

from test_gpu_q8_rows import TYPES, check

pytestmark = pytest.mark.gpu


def gated(gate, up):
    g = gate.double()
    return g / (1 + torch.exp(-g)) * up.double()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1e38, 2.3e38, 2.4e38, 3.3e38, None])
@pytest.mark.parametrize("up", [1e-30, 1e-3, 0.5, 1.0])
def test_gates_that_are_large(dtype, top, up):
    """Up to the largest finite one (None), alone among ordinary gates and in a row full of them: products that fp32 holds."""
    import paper_2401_12522_amd as bita
    g = torch.Generator(device="cuda").manual_seed(1)
    f, t = 500, TYPES[dtype]
    gate = torch.randn(2, f, device="cuda", generator=g)
    ups = up * torch.rand(2, f, device="cuda", generator=g)
    big = torch.finfo(t).max if top is None else top
    gate[0, 77] = big
    gate[1] = big * (0.5 + 0.5 * torch.rand(f, device="cuda", generator=g))
    gate[1, 3], ups[:, 77], ups[1, 3] = big, up, up
    gate, ups = gate.to(t), ups.to(t)
    v = gated(gate, ups)
    assert bool(torch.isfinite(v.float()).all())
    q, scale = bita.silu_mul_q8(torch.cat([gate, ups], 1).contiguous())
    check(q, scale, v)
    pairs = torch.stack([gate[:, :496].reshape(2, -1, 16), ups[:, :496].reshape(2, -1, 16)], 2).reshape(2, -1).contiguous()
    check(*bita.silu_mul_q8(pairs, tile=16), v[:, :496])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-45, 1e-43, 1e-41, 1e-39, 1.2e-38, 3e-38])
@pytest.mark.parametrize("up", [1e30, 1e34, 3e38])
def test_gates_that_are_subnormal(dtype, size, up):
    """Half of such a gate is no longer a multiple of the smallest number, and a large up brings the product back into the ordinary range."""
    import paper_2401_12522_amd as bita
    g = torch.Generator(device="cuda").manual_seed(2)
    f, t = 400, TYPES[dtype]
    gate = size * torch.randn(3, f, device="cuda", generator=g, dtype=torch.float64)
    ups = up * torch.rand(3, f, device="cuda", generator=g, dtype=torch.float64)
    gate[1, ::2], ups[1, ::2] = -1 - torch.rand(f // 2, device="cuda", generator=g, dtype=torch.float64), size * up
    gate[2, 5], ups[2, 5] = 60.0, size * up / 60
    gate, ups = gate.float().to(t), ups.float().to(t)
    q, scale = bita.silu_mul_q8(torch.cat([gate, ups], 1).contiguous())
    check(q, scale, gated(gate, ups))


def test_products_next_to_the_end_of_fp32():
    """A product that rounds to fp32's infinity is one, the next smaller one is a number: |v| at or above 2^128 - 2^103 or below it."""
    import paper_2401_12522_amd as bita
    g = torch.Generator(device="cuda").manual_seed(3)
    m, f = 4000, 24
    gate, ups = torch.randn(m, f, device="cuda", generator=g), torch.randn(m, f, device="cuda", generator=g)
    gate[:, 7] = 2 + 10 * torch.rand(m, device="cuda", generator=g)
    near = (torch.finfo(torch.float32).max / gated(gate[:, 7], torch.ones(m, device="cuda"))).float()
    step = torch.randint(-4, 5, (m,), device="cuda", generator=g, dtype=torch.int32)
    ups[:, 7] = (near.view(torch.int32) + step).view(torch.float32)
    v, limit = gated(gate, ups), 2.0 ** 128 - 2.0 ** 103
    beyond = v[:, 7] >= limit
    assert bool(((v[:, 7] / limit - 1).abs() > 1e-14).all())                # (none where doubles could not tell)
    assert 1000 < int(beyond.sum()) < 3000
    q, scale = bita.silu_mul_q8(torch.cat([gate, ups], 1).contiguous())
    assert torch.equal(torch.isnan(scale), beyond) and not q[beyond].any()
    check(q[~beyond], scale[~beyond], v[~beyond])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,f", [(3, 9000), (1500, 4100), (3, 20000), (3, 33000), (2, 70001)])
def test_long_rows_with_a_large_gate(m, f, dtype):
    """Rows of several groups of values a thread, and longer than a workgroup holds: a large gate in the last values, beside an ordinary row and an infinity."""
    import paper_2401_12522_amd as bita
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(m, 2 * f, device="cuda", generator=g)
    x[0, f - 2], x[0, 2 * f - 2] = 3e38, 0.25
    if m > 2:
        x[2, f - 1], x[2, 2 * f - 1] = float("inf"), 0.5
    x = x.to(TYPES[dtype])
    q, scale = bita.silu_mul_q8(x)
    rows = [r for r in range(m) if r != 2]
    check(q[rows], scale[rows], gated(x[rows, :f], x[rows, f:]))
    if m > 2:
        assert bool(torch.isnan(scale[2])) and not q[2].any()
