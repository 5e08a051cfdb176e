"""The tile kernel's outputs, which pass between the lanes of a wave on their way out (GPU): every tile form, fp32, bf16 and split sums,
row blocks and columns that end inside a tile.  Scales are powers of two and sums below 2^24, so that fp32 outputs are exact and a bf16 output
is the exact value's nearest."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _small(m, k, seed):
    import paper_2401_12522_amd as bita
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = bita.empty_q8(m, k)
    q.copy_(torch.randint(-11, 12, (m, k), device="cuda", generator=g))      # (11 * 11 * 131071 < 2^24)
    return q, 2.0 ** torch.randint(-3, 4, (m,), device="cuda", generator=g).float()


@pytest.mark.parametrize("m,n,k,rows,cols,split", [
    (898, 12646, 1507, 256, 256, False), (293, 32003, 400, 160, 256, False), (149, 34781, 21400, 160, 256, True), (520, 9000, 400, 128, 256, False),
    (300, 100, 131071, 128, 128, True), (1500, 130, 4001, 128, 128, True), (79, 79711, 905, 96, 192, False), (281, 22543, 515, 288, 128, False),
    (4244, 283, 5726, 288, 128, True)])
def test_every_value_arrives_in_its_place(m, n, k, rows, cols, split):
    import paper_2401_12522_amd as bita
    plan = bita.binding.gemm_q8_plan_info(m, n, k)
    assert (plan["rows"], plan["cols"], plan["splits"] > 1, plan["skinny"]) == (rows, cols, split, False), plan
    (a, sa), (w, sw) = _small(m, k, 1), _small(n, k, 2)
    packed = bita.pack_weight_q8(w)
    want = ((a.double() @ w.double().T) * sa.double()[:, None] * sw.double()).float()
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
        for _ in range(2):                                               # (the second over the first's values)
            bita.gemm_q8(a, sa, packed, sw, n, out=out)
            assert torch.equal(out, want.to(dtype))
