"""The norm that takes up the split sums of an 8-bit product, as a model's layers run it (GPU): the same bits as the product's own output
followed by the norm, in x, the integers and the scales."""
import ctypes as C

import pytest
import torch

from test_gpu_q8_gemm import codes

pytestmark = pytest.mark.gpu


class Sums(C.Structure):
    _fields_ = [("part", C.c_void_p), ("splits", C.c_int), ("row_scale", C.c_void_p), ("col_scale", C.c_void_p)]


def _library():
    """The two C++ functions behind the model's passes; the C interface has their parts only."""
    import paper_2401_12522_amd as bita
    L, vp, i32, i64 = bita.lib(), C.c_void_p, C.c_int32, C.c_int64
    product = L["_Z7gemm_q8PKalPKfilPKvS2_lPvmS5_ilP6SumsQ8P12ihipStream_t"]
    norm = L["_Z15norm_q8_of_sumsPfilRK6SumsQ8PKvfPalS_P12ihipStream_t"]
    product.restype, product.argtypes = C.c_int, [vp, i64, vp, i32, i64, vp, vp, i64, vp, C.c_size_t, vp, i32, i64, C.POINTER(Sums), vp]
    norm.restype, norm.argtypes = C.c_int, [vp, C.c_int, i64, C.POINTER(Sums), vp, C.c_float, vp, i64, vp, vp]
    return bita, product, norm


@pytest.mark.parametrize("m,d,k,skinny", [
    # few rows and many, one group of values a thread and two, sums of the kernel of few rows and of tiles, up to 8 splits
    (1, 256, 8192, True), (5, 256, 8192, True), (68, 4096, 11008, True), (68, 8192, 28672, True), (100, 16384, 20000, True), (300, 1024, 9001, False),
    (1024, 4096, 11008, False), (1100, 528, 20000, False), (2048, 5120, 13824, False)])
def test_the_same_bits_as_one_after_the_other(m, d, k, skinny):
    bita, product, norm = _library()
    plan = bita.binding.gemm_q8_plan_info(m, d, k)
    assert plan["skinny"] == skinny and plan["splits"] > 1, plan
    (a, sa), (w, sw) = codes(m, k, 1), codes(d, k, 2)
    if m > 4:
        a[1], sa[1] = 0, 0.0
        a[2], sa[2] = 0, float("nan")
    packed, g = bita.pack_weight_q8(w), torch.Generator(device="cuda").manual_seed(3)
    x0 = 100 * torch.randn(m, d, device="cuda", generator=g)
    gain = (1 + 0.2 * torch.randn(d, device="cuda", generator=g)).to(torch.bfloat16)
    x = x0.clone()
    q, scale = bita.norm_q8(x, gain, 1e-5, delta=bita.gemm_q8(a, sa, packed, sw, d))
    # the sums left where they are; the rows' scales are read and written in one buffer, as in a pass
    need = bita.lib().bita_gemm_q8_workspace_bytes(m, d, k)
    ws, out = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), torch.full((m, d), 3.0, device="cuda")
    left, x2, both, q2 = Sums(), x0.clone(), sa.clone(), bita.empty_q8(m, d)
    stream = torch.cuda.current_stream().cuda_stream
    assert product(a.data_ptr(), a.stride(0), both.data_ptr(), m, k, packed.data_ptr(), sw.data_ptr(), d, ws.data_ptr(), need, out.data_ptr(), 0, d, C.byref(left), stream) == 0
    assert left.splits == plan["splits"] and left.part == ws.data_ptr() and bool((out == 3.0).all())
    assert norm(x2.data_ptr(), m, d, C.byref(left), gain.data_ptr(), 1e-5, q2.data_ptr(), q2.stride(0), both.data_ptr(), stream) == 0
    torch.cuda.synchronize()
    live = ~torch.isnan(sa)
    assert torch.equal(x2[live], x[live]) and bool(torch.isnan(x2[~live]).all())
    assert torch.equal(q2, q) and torch.equal(both[live], scale[live]) and bool(torch.isnan(both[~live]).all()) and torch.equal(live, ~torch.isnan(scale))
