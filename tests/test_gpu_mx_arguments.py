"""What the Python calls of the small cache and the attention block refuse, and that a refused call writes nothing (GPU)."""
import numpy as np
import pytest
import torch

from test_gpu_kv_mx import i32, make, rows

pytestmark = pytest.mark.gpu


def parts():
    import paper_2401_12522_amd as bita
    tmpl = bita.TreeTemplate(np.array([-1, 0, 0], np.int32), np.zeros(3, np.uint8), 3, 0)
    t = dict(cache=make(2, 64, 2, 40, 4), q=rows((2, 3, 4, 64), 1, torch.bfloat16).cuda(), k=rows((2, 2, 3, 64), 2, torch.bfloat16).cuda(),
             v=rows((2, 2, 3, 64), 3, torch.bfloat16).cuda(), ctx=i32([5, 7]), start=i32([0, 3]))
    return bita, tmpl, t


CHANGES = {
    "half": lambda t: t.half(), "cpu": lambda t: t.cpu(), "short": lambda t: t[..., :-8], "fewer": lambda t: t[:1], "flat": lambda t: t.flatten(),
    "last axis not neighbours": lambda t: t.transpose(-1, -2).contiguous().transpose(-1, -2),
}


@pytest.mark.parametrize("which", ["q", "k", "v"])
@pytest.mark.parametrize("how", sorted(CHANGES))
def test_tree_attention_mx(which, how):
    bita, tmpl, t = parts()
    t[which] = CHANGES[how](t[which])
    out = torch.full((2, 3, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="wanted"):
        bita.tree_attention_mx(tmpl, t["q"], t["cache"], t["k"], t["v"], t["ctx"], 10, out=out)
    assert (out == 7).all()


def test_tree_attention_mx_other_arguments():
    bita, tmpl, t = parts()
    call = lambda ctx=t["ctx"], hint=10, **kw: bita.tree_attention_mx(tmpl, t["q"], t["cache"], t["k"], t["v"], ctx, hint, **kw)     # noqa: E731
    for bad in (dict(ctx=i32([5])), dict(ctx=torch.tensor([5, 7], device="cuda")), dict(token=i32([0, 1, 2])), dict(out=torch.empty((2, 3, 128), dtype=torch.bfloat16, device="cuda")),
                dict(prompt_k=t["k"], prompt_v=t["v"]), dict(workspace=torch.empty(64, device="cuda"))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(bita.BitaError, match="capacity"):
        call(hint=41)
    wide = torch.zeros((2, 2, 3, 68), dtype=torch.bfloat16, device="cuda")[..., :64]            # rows 136 bytes apart
    with pytest.raises(bita.BitaError, match="multiples"):
        bita.tree_attention_mx(tmpl, t["q"], t["cache"], wide, t["v"], t["ctx"], 10)
    assert call().shape == (2, 3, 256)


def test_cache_writes_and_reads():
    bita, tmpl, t = parts()
    before = t["cache"].k.clone()
    for bad in (dict(k=t["k"].half()), dict(v=t["v"].float()), dict(k=t["k"][:, :1]), dict(v=t["v"][:, :, :2]), dict(start=i32([0])), dict(start=t["start"].long()),
                dict(count=i32([1, 2, 3])), dict(path=i32([0, 1])), dict(cu_rows=i32([0, 1, 2]))):
        a = dict(dict(k=t["k"], v=t["v"], start=t["start"]), **bad)
        with pytest.raises(ValueError):
            bita.kv_write_mx(t["cache"], **a)
    with pytest.raises(bita.BitaError):                         # a path goes with rows by sequence
        bita.kv_write_mx(t["cache"], t["k"][0].transpose(0, 1), t["v"][0].transpose(0, 1), t["start"], path=i32([[0], [0]]), cu_rows=i32([0, 1, 2]))
    assert torch.equal(t["cache"].k, before)
    k = torch.full((2, 2, 9, 64), 5.0, device="cuda")
    for bad in (dict(k=k.double()), dict(k=k[:1]), dict(length=i32([1])), dict(start=i32([1])), dict(v=k.bfloat16())):
        with pytest.raises(ValueError):
            bita.kv_read_mx(t["cache"], **dict(dict(k=k, v=None, length=i32([1, 1])), **bad))
    with pytest.raises(bita.BitaError, match="overlap"):
        bita.kv_read_mx(t["cache"], k[:, :, :1].expand(2, 2, 9, 64), None, i32([1, 1]))
    assert (k == 5).all()


def test_caches_that_are_none():
    import paper_2401_12522_amd as bita
    for bad in (dict(bits=5), dict(head_dim=96), dict(smax=0), dict(block_table=i32([[0], [1]]), page_size=24), dict(block_table=i32([[0], [1]]), page_size=16),
                dict(block_table=i32([0, 1]), page_size=64), dict(k=torch.zeros(2, 2, 40, 32, device="cuda")), dict(v=torch.zeros((2, 2, 41, 32), dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            bita.KVCacheMX(**dict(dict(n_kv_heads=2, head_dim=64, batch=2, smax=40, bits=4), **bad))


def test_qk_norm_rope():
    import paper_2401_12522_amd as bita
    x = torch.randn(5, 8 * 64, device="cuda")
    cos, sin, pos = torch.ones(9, 32, device="cuda"), torch.zeros(9, 32, device="cuda"), i32([0, 1, 2, 3, 4])
    gain = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    good = dict(x=x, pos=pos, cos=cos, sin=sin, n_heads=4, n_kv_heads=2, q_gain=gain, k_gain=gain)
    bita.qk_norm_rope(**good)
    for bad in (dict(x=x.half()), dict(x=x[:, :500]), dict(pos=pos[:4]), dict(pos=pos.long()), dict(cos=cos.double()), dict(sin=sin[:8]), dict(q_gain=gain.float()),
                dict(k_gain=gain[:32]), dict(q=torch.empty(5, 4, 64, device="cuda")), dict(k=torch.empty((5, 4, 64), dtype=torch.bfloat16, device="cuda")), dict(n_heads=5)):
        with pytest.raises(ValueError):
            bita.qk_norm_rope(**dict(good, **bad))
    with pytest.raises(bita.BitaError, match="eps"):
        bita.qk_norm_rope(**good, eps=-1.0)


def test_prompt_attention():
    import paper_2401_12522_amd as bita
    q, k = torch.zeros((9, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((9, 2, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(q=q.float()), dict(k=k[:8]), dict(v=k[:, :, :32]), dict(cu_seqlens=torch.tensor([0, 9], device="cuda")), dict(q=q.cpu()), dict(q=q[0]),
                dict(out=torch.zeros((9, 128), dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            bita.prompt_attention(**dict(dict(q=q, k=k, v=k, cu_seqlens=i32([0, 9])), **bad))
    for bad in (dict(q=torch.zeros((9, 3, 64), dtype=torch.bfloat16, device="cuda")), dict(cu_seqlens=i32([0])), dict(q=torch.zeros((9, 4, 68), dtype=torch.bfloat16, device="cuda")[:, :, :64])):
        with pytest.raises(bita.BitaError):
            bita.prompt_attention(**dict(dict(q=q, k=k, v=k, cu_seqlens=i32([0, 9])), **bad))


def test_empty_calls():
    import paper_2401_12522_amd as bita
    none = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert bita.prompt_attention(none, none, none, i32([0, 0])).shape == (0, 128)
    cache = make(2, 64, 1, 8, 8)
    before = cache.k.clone()
    bita.kv_write_mx(cache, none, none, i32([0]), cu_rows=i32([0, 0]))
    k = torch.zeros((1, 2, 0, 64), device="cuda")
    bita.kv_read_mx(cache, k, k, i32([3]))
    assert torch.equal(cache.k, before)
    x = torch.zeros((0, 8 * 64), device="cuda")
    cos = torch.ones(9, 32, device="cuda")
    q, k, v = bita.qk_norm_rope(x, i32([]), cos, cos, 4, 2)
    assert q.shape == (0, 4, 64) and k.shape == v.shape == (0, 2, 64)
