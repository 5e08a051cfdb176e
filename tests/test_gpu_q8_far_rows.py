"""8-bit rows and products whose rows lie far apart (GPU): offsets that pass 32 bits, and the largest row stride of a product's activations."""
import pytest
import torch

from test_gpu_q8_gemm import check as check_product
from test_gpu_q8_gemm import codes
from test_gpu_q8_rows import check, rows

pytestmark = pytest.mark.gpu
FAR = (1 << 31) + 16


def _far(m, k, dtype):
    """A matrix whose rows are FAR elements apart, and the memory that holds it."""
    size = torch.empty((), dtype=dtype).element_size()
    memory = torch.empty(((m - 1) * FAR + k + 16) * size, dtype=torch.uint8, device="cuda").view(dtype)
    return memory.as_strided((m, k), (FAR, 1))


@pytest.mark.parametrize("call", ["rows", "norm", "gate"])
def test_rows_whose_offsets_pass_32_bits(call):
    import paper_2401_12522_amd as bita
    m, k = 3, 1003
    x, q = _far(m, 2 * k if call == "gate" else k, torch.bfloat16), _far(m, k, torch.int8)
    x.copy_(rows(m, x.shape[1], 1, torch.bfloat16))
    factor = None
    if call == "rows":
        q, s = bita.quantize_rows(x, q=q)
        v = x.double()
    elif call == "gate":
        q, s = bita.silu_mul_q8(x, q=q)
        g, u = x[:, :k].double(), x[:, k:].double()
        v = g / (1 + torch.exp(-g)) * u
    else:
        gain, delta = rows(1, k, 2, torch.bfloat16, 0.1)[0], _far(m, k, torch.float32)
        delta.copy_(rows(m, k, 3, torch.float32))
        h = (x.float() + delta).bfloat16()
        q, s = bita.norm_q8(x, gain, 1e-5, delta=delta, q=q)
        assert torch.equal(x, h)
        v, factor = h.double() * gain.double(), 1 / torch.sqrt(h.double().square().mean(1) + 1e-5)
    check(q.contiguous(), s, v, factor)


@pytest.mark.parametrize("m,n,k,skinny", [(3, 64, 500, True), (144, 500, 9001, True), (300, 600, 1601, False), (281, 22543, 515, False)])
def test_products_of_the_largest_row_stride(m, n, k, skinny):
    """Activations 8 MiB apart: the last row of a tile of 288 lies behind 2.4 GB."""
    import paper_2401_12522_amd as bita
    assert bita.binding.gemm_q8_plan_info(m, n, k)["skinny"] == skinny
    ld = 1 << 23
    (a0, sa), (w, sw) = codes(m, k, 1), codes(n, k, 2)
    a = torch.empty((m - 1) * ld + (k + 15) // 16 * 16, dtype=torch.int8, device="cuda").as_strided((m, k), (ld, 1))
    a.copy_(a0)
    packed = bita.pack_weight_q8(w)
    check_product(bita.gemm_q8(a, sa, packed, sw, n), a0, sa, w, sw)
    far = torch.empty((m - 1) * 65536 + n, dtype=torch.float32, device="cuda").as_strided((m, n), (65536, 1))
    check_product(bita.gemm_q8(a0, sa, packed, sw, n, out=far), a0, sa, w, sw)


def test_an_output_and_a_weight_whose_offsets_pass_32_bits():
    import paper_2401_12522_amd as bita
    for m, n, k in ((3, 300, 200), (40, 37, 200)):
        (a, sa), (w0, sw) = codes(m, k, 1), codes(n, k, 2)
        out = _far(m, n, torch.bfloat16) if m < 10 else torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
        w = w0 if m < 10 else _far(n, k, torch.int8).copy_(w0)
        check_product(bita.gemm_q8(a, sa, bita.pack_weight_q8(w), sw, n, out=out), a, sa, w0, sw)
