"""What the small-cache calls and the attention block around them refuse, before any device call (CPU only)."""
import ctypes as C

import pytest

P = 1 << 20        # a pointer that is never followed: multiple of 16
F32, BF16 = 0, 1


def _lib():
    from paper_2401_12522_amd import binding
    return binding.lib()


def _kv(**bad):
    from paper_2401_12522_amd import binding
    f = dict(k=P, v=P, k_scale=P, v_scale=P, bits=4, batch=2, n_kv_heads=2, head_dim=128, smax=100, block_table=None, page_size=0, n_pages=0, max_pages=0)
    f.update(bad)
    return C.byref(binding._KVMX(*f.values()))


class _Template:
    """A template handle without a device behind it: only its sizes are looked at before a call is refused."""

    def __init__(self, rows=3):
        self.buf = C.create_string_buffer(256)
        C.memmove(self.buf, (C.c_int32 * 7)(rows, rows, 0, 0, rows, 1, 1), 28)

    def pointer(self):
        return C.addressof(self.buf)


TMPL = _Template()
PAGED = dict(block_table=P, page_size=16, n_pages=20, max_pages=7)
WRITE = dict(kv={}, k=P, k_seq=512, k_head=256, k_row=128, v=P, v_seq=512, v_head=256, v_row=128, type=BF16, n=2, start=P, count=None, path=None, path_stride=0, cu=None,
             stream=None)
READ = dict(kv={}, k=P, k_seq=512, k_head=256, k_row=128, v=P, v_seq=512, v_head=256, v_row=128, type=BF16, n=2, start=None, length=P, stream=None)
ROPE = dict(x=P, type=F32, m=4, ldx=768, hq=2, hkv=2, hd=128, qg=P, kg=P, eps=1e-5, pos=P, cos=P, sin=P, max_pos=9, q=P, ldq=256, qh=128, k=P, ldk=256, kh=128, v=P, ldv=256,
            vh=128, stream=None)
TREE = dict(t=TMPL.pointer(), q=P, kv={}, k=P, k_seq=1024, k_head=512, k_row=128, v=P, v_seq=1024, v_head=512, v_row=128, pk=None, pv=None, n_prompt=0, ctx=P, token=None,
            heads=4, hint=50, ws=P, ws_bytes=1 << 30, out=P, stream=None)
PROMPT = dict(q=P, ldq=256, qh=64, k=P, ldk=128, kh=64, v=P, ldv=128, vh=64, cu=P, n_seqs=2, tokens=100, hq=4, hkv=2, hd=64, out=P, ldo=256, stream=None)
CALLS = dict(bita_kv_write_mx=WRITE, bita_kv_read_mx=READ, bita_qk_norm_rope=ROPE, bita_tree_attention_mx=TREE, bita_prompt_attention=PROMPT)


def _call(name, **bad):
    args = dict(CALLS[name], **bad)
    if "kv" in args and args["kv"] is not None:
        args["kv"] = _kv(**args["kv"])
    return getattr(_lib(), name)(*args.values())


KV_BAD = [(dict(k=None), -1), (dict(v_scale=None), -1), (dict(k=P + 8), -1), (dict(k_scale=P + 4), -1), (dict(bits=5), -4), (dict(head_dim=96), -4), (dict(batch=0), -1),
          (dict(smax=0), -1), (dict(n_kv_heads=0), -1), (dict(PAGED, page_size=24), -1), (dict(PAGED, page_size=8), -1), (dict(PAGED, n_pages=0), -1),
          (dict(PAGED, max_pages=6), -3)]


@pytest.mark.parametrize("name", ["bita_kv_write_mx", "bita_kv_read_mx", "bita_tree_attention_mx"])
@pytest.mark.parametrize("bad,code", KV_BAD)
def test_bad_caches(name, bad, code):
    assert _call(name, kv=bad) == code
    assert name.encode() in _lib().bita_last_error()


@pytest.mark.parametrize("name,bad,code", [
    ("bita_kv_write_mx", dict(kv=None), -1), ("bita_kv_write_mx", dict(k=None), -1), ("bita_kv_write_mx", dict(start=None), -1), ("bita_kv_write_mx", dict(type=2), -1),
    ("bita_kv_write_mx", dict(n=-1), -1), ("bita_kv_write_mx", dict(n=(1 << 27) + 1), -1), ("bita_kv_write_mx", dict(k_row=-128), -1), ("bita_kv_write_mx", dict(v_head=100), -4),
    ("bita_kv_write_mx", dict(k=P + 8), -4), ("bita_kv_write_mx", dict(path=P, path_stride=0), -1), ("bita_kv_write_mx", dict(path=P, path_stride=4, cu=P), -1),
    ("bita_kv_read_mx", dict(k=None, v=None), -1), ("bita_kv_read_mx", dict(length=None), -1), ("bita_kv_read_mx", dict(type=7), -1), ("bita_kv_read_mx", dict(n=-1), -1),
    ("bita_kv_read_mx", dict(k_seq=516), -4), ("bita_kv_read_mx", dict(v=P + 2), -4), ("bita_kv_read_mx", dict(k_row=0), -1), ("bita_kv_read_mx", dict(v_head=128), -1),
    ("bita_kv_read_mx", dict(k_seq=256), -1), ("bita_kv_read_mx", dict(v_row=64), -1),
    ("bita_qk_norm_rope", dict(x=None), -1), ("bita_qk_norm_rope", dict(pos=None), -1), ("bita_qk_norm_rope", dict(sin=None), -1), ("bita_qk_norm_rope", dict(k=None), -1),
    ("bita_qk_norm_rope", dict(type=3), -1), ("bita_qk_norm_rope", dict(m=-1), -1), ("bita_qk_norm_rope", dict(hq=0), -1), ("bita_qk_norm_rope", dict(max_pos=0), -1),
    ("bita_qk_norm_rope", dict(hd=80), -4), ("bita_qk_norm_rope", dict(ldx=760), -1), ("bita_qk_norm_rope", dict(ldx=772), -4), ("bita_qk_norm_rope", dict(ldq=-256), -1),
    ("bita_qk_norm_rope", dict(q=P + 8), -4), ("bita_qk_norm_rope", dict(qg=P + 4), -4), ("bita_qk_norm_rope", dict(cos=P + 4), -4), ("bita_qk_norm_rope", dict(vh=100), -4),
    ("bita_qk_norm_rope", dict(ldk=128), -1), ("bita_qk_norm_rope", dict(kh=64), -1), ("bita_qk_norm_rope", dict(eps=-1.0), -1), ("bita_qk_norm_rope", dict(eps=float("nan")), -1),
    ("bita_qk_norm_rope", dict(eps=float("inf")), -1),
    ("bita_tree_attention_mx", dict(t=None), -1), ("bita_tree_attention_mx", dict(q=None), -1), ("bita_tree_attention_mx", dict(kv=None), -1),
    ("bita_tree_attention_mx", dict(v=None), -1), ("bita_tree_attention_mx", dict(ctx=None), -1), ("bita_tree_attention_mx", dict(out=None), -1),
    ("bita_tree_attention_mx", dict(n_prompt=4), -1), ("bita_tree_attention_mx", dict(n_prompt=-1), -1), ("bita_tree_attention_mx", dict(heads=3), -1),
    ("bita_tree_attention_mx", dict(heads=0), -1), ("bita_tree_attention_mx", dict(hint=-1), -1), ("bita_tree_attention_mx", dict(hint=101), -3),
    ("bita_tree_attention_mx", dict(q=P + 8), -4), ("bita_tree_attention_mx", dict(k_row=132), -4), ("bita_tree_attention_mx", dict(v_seq=-8), -1),
    ("bita_tree_attention_mx", dict(heads=1 << 17), -4), ("bita_tree_attention_mx", dict(kv=dict(smax=100000), hint=100000, ws_bytes=64), -3),
    ("bita_tree_attention_mx", dict(kv=dict(smax=100000), hint=100000, ws=None), -3),
    ("bita_prompt_attention", dict(q=None), -1), ("bita_prompt_attention", dict(cu=None), -1), ("bita_prompt_attention", dict(out=None), -1),
    ("bita_prompt_attention", dict(n_seqs=0), -1), ("bita_prompt_attention", dict(tokens=-1), -1), ("bita_prompt_attention", dict(hq=5), -1), ("bita_prompt_attention", dict(hd=32), -4),
    ("bita_prompt_attention", dict(ldo=248), -1), ("bita_prompt_attention", dict(ldq=-8), -1), ("bita_prompt_attention", dict(ldk=132), -4), ("bita_prompt_attention", dict(v=P + 4), -4),
    ("bita_prompt_attention", dict(tokens=(1 << 31) - 1, hq=64, hkv=64, ldo=4096), -4),
])
def test_refused_with_a_message(name, bad, code):
    assert _call(name, **bad) == code
    assert name.encode() in _lib().bita_last_error()


def test_nothing_to_do_is_no_error():
    assert _call("bita_kv_write_mx", n=0) == 0 and _call("bita_kv_read_mx", n=0) == 0
    assert _call("bita_qk_norm_rope", m=0) == 0 and _call("bita_prompt_attention", tokens=0) == 0


def test_sizes_of_workspaces_and_plans():
    L, out = _lib(), (C.c_int32 * 4)()
    assert L.bita_tree_attention_mx_workspace_bytes(1, 1, 4, 3, 128, 4, 100, 0) == 0 and b"workspace_bytes" in L.bita_last_error()
    assert L.bita_tree_attention_mx_plan_info(1, 1, 4, 4, 128, 6, 100, 0, out) == -4
    assert L.bita_tree_attention_mx_plan_info(1, 1, 4, 4, 128, 4, 100, 0, None) == -1
    for n, r, hq, hkv, hd, hint, prefix in ((1, 1, 1, 1, 64, 0, 0), (1, 1, 64, 8, 128, 131072, 0), (32, 1, 64, 8, 128, 8192, 0), (4, 68, 64, 8, 128, 4096, 16), (3, 512, 7, 7, 64, 9, 5)):
        assert L.bita_tree_attention_mx_plan_info(n, r, hq, hkv, hd, 4, hint, prefix, out) == 0
        splits, queries, waves, wgs = out
        chunks = -(-hint // 32) + -(-prefix // 32) + -(-r // 32)
        assert 1 <= splits <= max(1, chunks) and waves > 0 and wgs == n * hkv * -(-r * (hq // hkv) // queries) * splits
        need = L.bita_tree_attention_mx_workspace_bytes(n, r, hq, hkv, hd, 4, hint, prefix)
        assert need >= (n * r * hq * splits * (hd + 2) * 4 if splits > 1 else 0)
