"""Gating at the ends of the gates' range (GPU): gates whose exponent passes fp32, against silu(g) u in 64 bits.  Every integer has to be
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
