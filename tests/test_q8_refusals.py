"""What the 8-bit linear layers refuse, before any device call (CPU only)."""
import pytest

P = 1 << 20        # a pointer that is never followed: multiple of 16
F32, BF16 = 0, 1


def _lib():
    from paper_2401_12522_amd import binding
    return binding.lib()


def _call(name, good, **bad):
    args = dict(good, **bad)
    return getattr(_lib(), name)(*args.values())


ROWS = dict(x=P, x_type=F32, m=4, k=64, ldx=64, q=P, ldq=64, scale=P, stream=None)
NORM = dict(x=P, x_type=F32, m=4, d=64, ldx=64, delta=P, delta_type=BF16, ld_delta=64, gain=P, eps=1e-5, total=P, ld_total=64, q=P, ldq=64,
            scale=P, stream=None)
GATE = dict(x=P, x_type=BF16, m=4, f=64, ldx=128, tile=16, q=P, ldq=64, scale=P, stream=None)
PACK = dict(src=P, n=32, k=64, ld=64, dst=P, total=64, tile0=0, stride=1, stream=None)
GEMM = dict(a=P, lda=64, a_scale=P, m=4, k=64, w=P, w_scale=P, n=64, ws=None, ws_bytes=0, out=P, out_type=F32, ldo=64, stream=None)


@pytest.mark.parametrize("name,good,bad,code", [
    ("bita_quantize_rows", ROWS, dict(x=None), -1), ("bita_quantize_rows", ROWS, dict(q=None), -1), ("bita_quantize_rows", ROWS, dict(scale=None), -1),
    ("bita_quantize_rows", ROWS, dict(x_type=2), -1), ("bita_quantize_rows", ROWS, dict(m=0), -1), ("bita_quantize_rows", ROWS, dict(k=0), -1),
    ("bita_quantize_rows", ROWS, dict(ldx=63), -1), ("bita_quantize_rows", ROWS, dict(ldq=63), -1),
    ("bita_quantize_rows", ROWS, dict(k=131072, ldx=131072, ldq=131072), -4),
    ("bita_norm_q8", NORM, dict(x=None), -1), ("bita_norm_q8", NORM, dict(gain=None), -1), ("bita_norm_q8", NORM, dict(total=None), -1),
    ("bita_norm_q8", NORM, dict(delta_type=7), -1), ("bita_norm_q8", NORM, dict(ld_delta=60), -1), ("bita_norm_q8", NORM, dict(ld_total=60), -1),
    ("bita_norm_q8", NORM, dict(ld_total=80), -1), ("bita_norm_q8", NORM, dict(eps=-1.0), -1), ("bita_norm_q8", NORM, dict(eps=float("nan")), -1),
    ("bita_norm_q8", NORM, dict(d=16385, ldx=16400, ld_delta=16400, ld_total=16400, ldq=16400), -4), ("bita_norm_q8", NORM, dict(m=-1), -1),
    ("bita_silu_mul_q8", GATE, dict(x=None), -1), ("bita_silu_mul_q8", GATE, dict(ldx=127), -1), ("bita_silu_mul_q8", GATE, dict(tile=8), -1),
    ("bita_silu_mul_q8", GATE, dict(f=40), -1), ("bita_silu_mul_q8", GATE, dict(f=131088, ldx=1 << 20, ldq=1 << 20), -4),
    ("bita_pack_weight_q8", PACK, dict(src=None), -1), ("bita_pack_weight_q8", PACK, dict(dst=P + 8), -1), ("bita_pack_weight_q8", PACK, dict(ld=63), -1),
    ("bita_pack_weight_q8", PACK, dict(tile0=3), -1), ("bita_pack_weight_q8", PACK, dict(stride=4), -1), ("bita_pack_weight_q8", PACK, dict(stride=0), -1),
    ("bita_pack_weight_q8", PACK, dict(n=20), -4), ("bita_pack_weight_q8", PACK, dict(k=131072, ld=131072), -4),
    ("bita_gemm_q8", GEMM, dict(a=None), -1), ("bita_gemm_q8", GEMM, dict(a_scale=None), -1), ("bita_gemm_q8", GEMM, dict(w=None), -1),
    ("bita_gemm_q8", GEMM, dict(w_scale=None), -1), ("bita_gemm_q8", GEMM, dict(out=None), -1), ("bita_gemm_q8", GEMM, dict(m=0), -1),
    ("bita_gemm_q8", GEMM, dict(n=0), -1), ("bita_gemm_q8", GEMM, dict(k=0), -1), ("bita_gemm_q8", GEMM, dict(out_type=3), -1),
    ("bita_gemm_q8", GEMM, dict(ldo=63), -1), ("bita_gemm_q8", GEMM, dict(lda=72), -1), ("bita_gemm_q8", GEMM, dict(lda=48), -1),
    ("bita_gemm_q8", GEMM, dict(out=P + 2), -1), ("bita_gemm_q8", GEMM, dict(out=P + 1, out_type=BF16), -1), ("bita_gemm_q8", GEMM, dict(lda=(1 << 23) + 16), -4),
    ("bita_gemm_q8", GEMM, dict(m=68, k=28672, lda=28672, n=8192, ldo=8192), -3), ("bita_gemm_q8", GEMM, dict(m=68, k=28672, lda=28672, n=8192, ldo=8192, ws=P, ws_bytes=1 << 16), -3),
    ("bita_gemm_q8", GEMM, dict(a=P + 8), -1), ("bita_gemm_q8", GEMM, dict(k=131072, lda=131088), -4),
])
def test_refused_with_a_message(name, good, bad, code):
    assert _call(name, good, **bad) == code
    assert name.encode() in _lib().bita_last_error()


@pytest.mark.parametrize("name,good,bad,code", [
    # strides whose last tile's number wraps around 64 bits
    ("bita_pack_weight_q8", PACK, dict(stride=(1 << 63) - 1), -1), ("bita_pack_weight_q8", dict(PACK, n=80), dict(stride=1 << 62), -1),
    ("bita_pack_weight_q8", PACK, dict(tile0=(1 << 63) - 1), -1),
    ("bita_pack_weight_q8", PACK, dict(n=(1 << 26) + 16, total=1 << 27), -4), ("bita_gemm_q8", GEMM, dict(n=(1 << 26) + 1, ldo=1 << 27), -4),
    ("bita_norm_q8", NORM, dict(eps=float("inf")), -1),
])
def test_refused_beyond_a_launch(name, good, bad, code):
    test_refused_with_a_message(name, good, bad, code)


def test_workspace_of_refused_sizes():
    L = _lib()
    assert L.bita_gemm_q8_workspace_bytes(4, (1 << 26) + 1, 4096) == L.bita_gemm_q8_workspace_bytes(4, 64, 131072) == 0


def test_packed_sizes():
    L = _lib()
    assert L.bita_packed_q8_bytes(32, 688) == 2 * 6 * 2048
    assert L.bita_packed_q8_bytes(33, 1) == 3 * 2048
    assert L.bita_packed_q8_bytes(0, 5) == L.bita_packed_q8_bytes(5, 0) == 0


def test_refusals_of_an_8_bit_model():
    import ctypes as C
    import paper_2401_12522_amd as bita
    L = bita.lib()
    cfg = bita.binding._Config(1, 64, 1, 1, 64, 16, 16, 0, 0, 8, 1e-5, 1e4)
    w, sq, handle = bita.binding._Weights(), bita.binding._ScalesQ8(), C.c_void_p()
    assert L.bita_model_create_q8(C.byref(cfg), C.byref(w), None, C.byref(handle)) == -1
    assert L.bita_model_create_q8(C.byref(cfg), C.byref(w), C.byref(sq), C.byref(handle)) == -1
    one = (C.c_void_p * 1)(1 << 20)
    none = (C.c_void_p * 1)(None)
    for n in ("wqkv", "wo", "w_gate_up", "w_down"):
        setattr(sq, n, one)
    sq.wo = none
    assert L.bita_model_create_q8(C.byref(cfg), C.byref(w), C.byref(sq), C.byref(handle)) == -1
    sq.wo = one
    assert L.bita_model_create_q8(C.byref(cfg), C.byref(w), C.byref(sq), C.byref(handle)) == -1         # (no weights)
    wide = bita.binding._Config(1, 64, 1, 1, 64, 131072, 16, 0, 0, 8, 1e-5, 1e4)
    assert L.bita_model_create_q8(C.byref(wide), C.byref(w), C.byref(sq), C.byref(handle)) == -4
    assert not handle
