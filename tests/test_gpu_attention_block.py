"""The attention block of a decoder with a small cache, its calls one behind the other as a layer makes them (GPU): prompts of
several sequences (norm and rotation, attention over the packed rows, the rows into the cache), then steps of a token tree whose accepted rows follow.
Every call is checked against float64 from the bf16 tensors that the one before it left, and the cache's contents against the rows' rounding."""
import pytest
import torch

import mx_reference as ref
from test_gpu_kv_mx import i32, make, slots
from test_gpu_prompt_attention import expected as prompt_expected, near, starts
from test_gpu_qk_norm_rope import near as rope_near, reference, table
from test_gpu_tree_attention_mx import expected, template

pytestmark = pytest.mark.gpu


def cached(cache, ctx):
    """Values of the cache's slots, those at and behind a sequence's length as zeros."""
    k, v = (ref.values(ref.unpack(slots(cache, c), cache.bits), slots(cache, s), cache.bits) for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
    return k, v, [k[b, :, :n] for b, n in enumerate(ctx)]


@pytest.mark.parametrize("bits,hq,hkv,hd,page,dtype", [(4, 4, 2, 64, 16, torch.bfloat16), (8, 8, 1, 128, 0, torch.float32), (4, 6, 6, 128, 64, torch.bfloat16)])
def test_prompts_then_steps(bits, hq, hkv, hd, page, dtype):
    import paper_2401_12522_amd as bita
    g = torch.Generator().manual_seed(bits + hd)
    lens, smax, R, masks, P = [45, 1, 130], 200, 9, 3, 4
    n, cu = len(lens), starts(lens)
    cache = make(hkv, hd, n, smax, bits, page)
    cos, sin = table(smax + 16, hd)
    gains = [(1 + 0.2 * torch.randn(hd, generator=g)).to(torch.bfloat16) for _ in range(2)]
    pk, pv = (torch.randn(hkv, P, hd, generator=g).to(torch.bfloat16) for _ in range(2))

    def rotated(m, pos):
        x = torch.randn(m, (hq + 2 * hkv) * hd, generator=g).to(dtype)
        q, k, v = bita.qk_norm_rope(x.cuda(), pos.int().cuda(), cos.cuda(), sin.cuda(), hq, hkv, gains[0].cuda(), gains[1].cuda(), 1e-5)
        wq, wk, wv = reference(x, hq, hkv, hd, *gains, 1e-5, pos, cos, sin)
        rope_near(q, wq)
        rope_near(k, wk)
        assert torch.equal(v.cpu(), wv)
        return q, k, v

    q, k, v = rotated(cu[-1], torch.cat([torch.arange(x) for x in lens]))
    near(bita.prompt_attention(q, k, v, i32(cu)), *prompt_expected(q.cpu(), k.cpu(), v.cpu(), cu))
    bita.kv_write_mx(cache, k, v, i32([0] * n), cu_rows=i32(cu))
    rows_k = [ref.rounded(k[a:b].cpu().transpose(0, 1), bits) for a, b in zip(cu, cu[1:])]
    tmpl, seen, is_mask = template(R, masks, 1)
    depth = seen.sum(1) - 1
    ctx = list(lens)
    for step, acc in enumerate(([3, 1, 2], [1, 2, 3], [2, 2, 1])):
        path = torch.zeros(n, 3, dtype=torch.int32)
        for b in range(n):
            node = int((depth[: R - masks]).argmax())
            chain = [r for r in range(R - masks) if seen[node, r]]
            acc[b] = min(acc[b], len(chain))
            path[b, : acc[b]] = torch.tensor(chain[: acc[b]])
        pos = torch.tensor(ctx)[:, None] + depth[None]
        q, k, v = rotated(n * R, pos.flatten())
        k, v = (t.unflatten(0, (n, R)).transpose(1, 2) for t in (k, v))
        q = q.view(n, R, hq, hd)
        out = bita.tree_attention_mx(tmpl, q, cache, k, v, i32(ctx), max(ctx), pk.cuda(), pv.cuda())
        ck, cv, _ = cached(cache, ctx)
        near(out, *expected(q.cpu(), ck, cv, k.cpu(), v.cpu(), ctx, seen, is_mask, pk, pv))
        bita.kv_write_mx(cache, k, v, i32(ctx), i32(acc), path=path.cuda())
        for b in range(n):
            rows_k[b] = torch.cat([rows_k[b], ref.rounded(k[b].cpu()[:, path[b, : acc[b]].long()], bits)], 1)
            ctx[b] += acc[b]
        _, _, held = cached(cache, ctx)
        for b in range(n):
            assert torch.equal(held[b], rows_k[b])
    k, v = (torch.zeros(n, hkv, max(ctx), hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bita.kv_read_mx(cache, k, v, i32(ctx))
    for b in range(n):
        assert torch.equal(k[b, :, : ctx[b]].cpu().double(), rows_k[b]) and not k[b, :, ctx[b]:].any()


def test_small_cache_agrees_with_the_bf16_one():
    """tree_attention over a bf16 cache that holds what the 8-bit one reads back gives the same as tree_attention_mx, within both
    roundings (two of half a step of bf16 for each side's, on the sum of |p v|)."""
    import paper_2401_12522_amd as bita
    from test_gpu_tree_attention_mx import case
    call, (out, tol), (cache, q, kr, vr, ck, cv, tmpl, seen, is_mask) = case(2, 20, 4, 8, 2, 128, 8, [300, 77], P=0, smax=320)
    k, v = (torch.zeros(2, 2, 320, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bita.kv_read_mx(cache, k, v, i32([300, 77]))
    wide = bita.tree_attention(tmpl, q.cuda(), k, v, kr.cuda(), vr.cuda(), None, None, i32([300, 77]), 300)
    near(wide, out, tol)
    near(call(), out, tol)


def test_two_streams_and_another_thread():
    """The calls on two streams at once, from two threads, each with tensors of its own, give what they give alone."""
    import threading
    import paper_2401_12522_amd as bita
    from test_gpu_kv_mx import rows
    from test_gpu_tree_attention_mx import case

    def work(seed):
        call, _, parts = case(2, 1, 0, 8, 2, 128, 4, [3000, 1000], 16, seed=seed)
        cache, q = parts[0], parts[1]
        p = [rows((500, h, 64), seed + i, torch.bfloat16).cuda() for i, h in enumerate((4, 2, 2))]
        back = torch.zeros(2, 2, 64, 128, dtype=torch.bfloat16, device="cuda")

        def run():
            bita.kv_read_mx(cache, back, None, i32([64, 64]))
            return call(), bita.prompt_attention(*p, i32([0, 250, 500])), back.clone()
        return run
    jobs = [work(s) for s in (1, 2)]
    alone = [j() for j in jobs]
    torch.cuda.synchronize()
    got, failed = [None, None], []

    def thread(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(5):
                    got[i] = jobs[i]()
            s.synchronize()
        except Exception as e:                                    # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=thread, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for a, b in zip(alone, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
