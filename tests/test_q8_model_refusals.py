"""More of what the creation of an 8-bit model refuses, before any device call (CPU only)."""
import ctypes as C

import paper_2401_12522_amd as bita

NAMES = ("wqkv", "wo", "w_gate_up", "w_down")


def test_a_missing_place_for_the_handle_is_refused():
    """Everything else is in order, so that nothing else refuses it; the pointers are never followed."""
    L = bita.lib()
    cfg = bita.binding._Config(1, 64, 1, 1, 64, 16, 16, 0, 0, 8, 1e-5, 1e4)
    one = (C.c_void_p * 1)(1 << 20)
    w, scales = bita.binding._Weights(), bita.binding._ScalesQ8()
    for n in ("attn_norm", "ffn_norm") + NAMES:
        setattr(w, n, one)
    for n in ("tok_emb", "final_norm", "lm_head"):
        setattr(w, n, 1 << 20)
    for n in NAMES:
        setattr(scales, n, one)
    assert L.bita_model_create_q8(C.byref(cfg), C.byref(w), C.byref(scales), None) == -1
    assert b"bita_model_create_q8" in L.bita_last_error()
