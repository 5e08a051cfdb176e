"""Norm and rotation of queries and keys (GPU) against float64 on the CPU.
Tolerance: half a step of bf16 for the rounding; in fp32 a sum of squares (at most 11 roundings deep), a quotient, a root and three products before
the rotation, whose two products and sum are three more: under 32 units of 2^-24 of the two values rotated."""
import pytest
import torch

pytestmark = pytest.mark.gpu
HALF = torch.finfo(torch.bfloat16).eps / 2


def table(max_pos, hd, theta=10000.0):
    a = torch.arange(max_pos, dtype=torch.float64)[:, None] * theta ** (-2 * torch.arange(hd // 2, dtype=torch.float64) / hd)
    return a.cos().float(), a.sin().float()


def reference(x, hq, hkv, hd, qg, kg, eps, pos, cos, sin):
    m = x.shape[0]
    x = x.double().view(m, hq + 2 * hkv, hd)
    out = []
    for lo, hi, g in ((0, hq, qg), (hq, hq + hkv, kg)):
        h = x[:, lo:hi]
        if g is not None:
            h = h / (h.square().mean(-1, keepdim=True) + eps).sqrt() * g.double()
        c, s = cos.double()[pos][:, None], sin.double()[pos][:, None]
        a, b = h[..., : hd // 2], h[..., hd // 2:]
        y = torch.cat([a * c - b * s, b * c + a * s], -1)
        size = (a.abs() + b.abs()).repeat(1, 1, 2)
        out.append((y, HALF * y.abs() + 32 * 2.0 ** -24 * (1 + HALF) * size))
    v = x[:, hq + hkv:]
    return out[0], out[1], v.to(torch.bfloat16)


def data(m, hq, hkv, hd, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(m, (hq + 2 * hkv) * hd, generator=g) * torch.exp(torch.randn(m, 1, generator=g))).to(dtype)
    gains = [(1 + 0.3 * torch.randn(hd, generator=g)).to(torch.bfloat16) for _ in range(2)]
    return x, gains


def near(got, want):
    y, tol = want
    assert ((got.cpu().double() - y).abs() <= tol).all()


@pytest.mark.parametrize("m,hq,hkv,hd,dtype,norm", [
    (1, 32, 32, 128, torch.float32, True), (1, 4, 2, 64, torch.bfloat16, True), (7, 4, 4, 64, torch.float32, False), (68, 64, 8, 128, torch.float32, True),
    (33, 12, 4, 64, torch.bfloat16, True), (5, 6, 2, 128, torch.bfloat16, False), (300, 1, 1, 128, torch.bfloat16, True), (3, 71, 71, 64, torch.float32, True)])
def test_against_float64(m, hq, hkv, hd, dtype, norm):
    import paper_2401_12522_amd as bita
    x, (qg, kg) = data(m, hq, hkv, hd, dtype)
    if not norm:
        qg = kg = None
    cos, sin = table(5000, hd)
    pos = torch.randint(0, 5000, (m,), generator=torch.Generator().manual_seed(1))
    up = lambda t: None if t is None else t.cuda()                # noqa: E731
    q, k, v = bita.qk_norm_rope(x.cuda(), pos.int().cuda(), cos.cuda(), sin.cuda(), hq, hkv, up(qg), up(kg), eps=1e-5)
    wq, wk, wv = reference(x, hq, hkv, hd, qg, kg, 1e-5, pos, cos, sin)
    near(q, wq)
    near(k, wk)
    assert torch.equal(v.cpu(), wv)


def test_columns_of_the_product_in_place_and_strided_outputs():
    import paper_2401_12522_amd as bita
    m, hq, hkv, hd = 37, 6, 2, 128
    x, (qg, kg) = data(m, hq, hkv, hd, torch.bfloat16, 2)
    cos, sin = table(64, hd)
    pos = torch.arange(m)
    wq, wk, _ = reference(x, hq, hkv, hd, qg, kg, 1e-6, pos, cos, sin)
    args = (pos.int().cuda(), cos.cuda(), sin.cuda(), hq, hkv, qg.cuda(), kg.cuda(), 1e-6)
    y = x.cuda()
    heads = y.view(m, hq + 2 * hkv, hd)
    q, k, v = bita.qk_norm_rope(y, *args, q=heads[:, :hq], k=heads[:, hq:hq + hkv])
    near(q, wq)
    near(k, wk)
    assert torch.equal(v.cpu().reshape(m, -1), x[:, (hq + hkv) * hd:]) and v.data_ptr() == heads[:, hq + hkv:].data_ptr()
    # [heads][rows][hd] outputs, rows of x further apart than they are long
    wide = torch.full((m, (hq + 2 * hkv) * hd + 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, : -64] = x.cuda()
    qo, ko, vo = (torch.zeros((n, m + 1, hd), dtype=torch.bfloat16, device="cuda") for n in (hq, hkv, hkv))
    bita.qk_norm_rope(wide[:, : -64], *args, q=qo[:, :m].transpose(0, 1), k=ko[:, :m].transpose(0, 1), v=vo[:, :m].transpose(0, 1))
    near(qo[:, :m].transpose(0, 1), wq)
    near(ko[:, :m].transpose(0, 1), wk)
    assert torch.equal(vo[:, :m].transpose(0, 1).cpu().reshape(m, -1), x[:, (hq + hkv) * hd:])
    assert not qo[:, m].any() and not ko[:, m].any() and not vo[:, m].any()


def test_positions_outside_the_table_take_its_ends():
    import paper_2401_12522_amd as bita
    x, (qg, kg) = data(4, 2, 1, 64, torch.float32, 3)
    cos, sin = table(9, 64)
    pos = torch.tensor([-1, -2 ** 31, 9, 2 ** 31 - 1])
    q, k, _ = bita.qk_norm_rope(x.cuda(), pos.int().cuda(), cos.cuda(), sin.cuda(), 2, 1, qg.cuda(), kg.cuda())
    wq, wk, _ = reference(x, 2, 1, 64, qg, kg, 1e-5, pos.clamp(0, 8), cos, sin)
    near(q, wq)
    near(k, wk)


@pytest.mark.parametrize("size", [1e-40, 1e-25, 1e-19, 1e18, 1e25, 1e37])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_squares_beyond_fp32(size, eps):
    """Heads whose squares leave fp32's range are normed all the same."""
    import paper_2401_12522_amd as bita
    x, (qg, kg) = data(5, 2, 2, 128, torch.float32, 4)
    x = x.div(x.abs().max()) * size
    cos, sin = table(9, 128)
    pos = torch.arange(5)
    q, k, _ = bita.qk_norm_rope(x.cuda(), pos.int().cuda(), cos.cuda(), sin.cuda(), 2, 2, qg.cuda(), kg.cuda(), eps=eps)
    (yq, tq), (yk, tk), _ = reference(x, 2, 2, 128, qg, kg, torch.tensor(eps).float().double(), pos, cos, sin)
    tiny = 2.0 ** -133 + 2.0 ** -148                               # below the normal numbers: half a step of bf16's subnormals, and of fp32's where they are rotated
    near(q, (yq, tq + tiny))
    near(k, (yk, tk + tiny))


def test_a_head_that_is_no_number_stays_its_own():
    import paper_2401_12522_amd as bita
    x, (qg, kg) = data(3, 4, 2, 64, torch.float32, 5)
    x.view(3, 8, 64)[1, 2, 7] = float("nan")
    x.view(3, 8, 64)[2, 5, 3] = float("inf")
    x.view(3, 8, 64)[0, 0] = 0.0
    cos, sin = table(9, 64)
    pos = torch.arange(3)
    q, k, _ = bita.qk_norm_rope(x.cuda(), pos.int().cuda(), cos.cuda(), sin.cuda(), 4, 2, qg.cuda(), kg.cuda())
    q, k = q.cpu(), k.cpu()
    assert q[1, 2].isnan().all() and k[2, 1].isnan().any() and not q[0, 0].any()
    q[1, 2], k[2, 1] = 0, 0
    assert q.isfinite().all() and k.isfinite().all()


def test_many_rows():
    """More rows than a launch has workgroups for."""
    import paper_2401_12522_amd as bita
    m, hd = (1 << 20) + 777, 64
    x, (qg, kg) = data(m, 1, 1, hd, torch.bfloat16, 6)
    cos, sin = table(64, hd)
    pos = torch.arange(m) % 64
    q, k, _ = bita.qk_norm_rope(x.cuda(), pos.int().cuda(), cos.cuda(), sin.cuda(), 1, 1, qg.cuda(), kg.cuda())
    wq, wk, _ = reference(x, 1, 1, hd, qg, kg, 1e-5, pos, cos, sin)
    near(q, wq)
    near(k, wk)
