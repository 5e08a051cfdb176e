"""Attention over the 4- and 8-bit cache (GPU) against float64 on the CPU; the tolerance is worked out in mx_reference.attention."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import synth
from test_gpu_kv_mx import i32, make, rows

pytestmark = pytest.mark.gpu
BITS = pytest.mark.parametrize("bits", [4, 8])


def template(rows_, masks=0, seed=0):
    """A random tree of rows_ rows, the last `masks` a group on its root: (handle, visible [R][R], is_mask [R])."""
    import paper_2401_12522_amd as bita
    t = rows_ - masks
    parent = list(synth.random_tree(t, 4, seed)) if t > 1 else [-1]
    parent += [0] + list(range(t, rows_ - 1)) if masks else []
    seen = torch.zeros(rows_, rows_, dtype=torch.bool)
    for i, p in enumerate(parent):
        if p >= 0:
            seen[i] = seen[p]
        seen[i, i] = True
    is_mask = torch.arange(rows_) >= t
    return bita.TreeTemplate(np.array(parent, np.int32), is_mask.numpy().astype(np.uint8), t, masks), seen, is_mask


def filled(hkv, hd, n, smax, bits, page, seed):
    """A cache with every slot written, and its values [n][hkv][smax][hd]."""
    import paper_2401_12522_amd as bita
    cache = make(hkv, hd, n, smax, bits, page, seed)
    k, v = rows((n, hkv, smax, hd), seed + 1, torch.bfloat16), rows((n, hkv, smax, hd), seed + 2, torch.bfloat16)
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), i32([0] * n))
    return cache, ref.rounded(k, bits), ref.rounded(v, bits)


def expected(q, ck, cv, kr, vr, ctx, seen, is_mask, pk=None, pv=None):
    """[n][R][hq][hd] and its tolerance."""
    n, R, hq, hd = q.shape
    hkv = kr.shape[1]
    out, tol = torch.zeros(2, n, R, hq, hd, dtype=torch.float64)
    P = 0 if pk is None else pk.shape[1]
    for b in range(n):
        vis = torch.ones(R, P + ctx[b] + R, dtype=torch.bool)
        vis[:, :P] = is_mask[:, None]
        vis[:, P + ctx[b]:] = seen
        for h in range(hq):
            g = h // (hq // hkv)
            k = torch.cat(([pk[g].double()] if P else []) + [ck[b, g, : ctx[b]], kr[b, g].double()])
            v = torch.cat(([pv[g].double()] if P else []) + [cv[b, g, : ctx[b]], vr[b, g].double()])
            out[b, :, h], tol[b, :, h] = ref.attention(q[b, :, h].double(), k, v, vis)
    return out, tol


def near(got, out, tol):
    off = (got.cpu().double().view(out.shape) - out).abs()
    assert (off <= tol).all(), float((off / tol).max())


def case(n, R, masks, hq, hkv, hd, bits, ctx, page=0, P=0, seed=0, smax=None):
    import paper_2401_12522_amd as bita
    tmpl, seen, is_mask = template(R, masks, seed)
    smax = smax or max(max(ctx), 1)
    cache, ck, cv = filled(hkv, hd, n, smax, bits, page, seed + 10)
    q, kr, vr = rows((n, R, hq, hd), seed + 20, torch.bfloat16), rows((n, hkv, R, hd), seed + 21, torch.bfloat16), rows((n, hkv, R, hd), seed + 22, torch.bfloat16)
    pk = pv = None
    if P:
        pk, pv = rows((hkv, P, hd), seed + 23, torch.bfloat16), rows((hkv, P, hd), seed + 24, torch.bfloat16)
    up = lambda t: None if t is None else t.cuda()                # noqa: E731
    call = lambda **kw: bita.tree_attention_mx(tmpl, q.cuda(), cache, kr.cuda(), vr.cuda(), i32(ctx), max(ctx), up(pk), up(pv), **kw)      # noqa: E731
    return call, expected(q, ck, cv, kr, vr, ctx, seen, is_mask, pk, pv), (cache, q, kr, vr, ck, cv, tmpl, seen, is_mask)


@BITS
@pytest.mark.parametrize("n,R,masks,hq,hkv,hd,ctx,page,P", [
    (1, 1, 0, 4, 4, 64, [0], 0, 0),                               # nothing cached: the row itself
    (1, 1, 0, 4, 2, 128, [1], 0, 0),
    (2, 1, 0, 8, 8, 128, [31, 33], 0, 0),
    (3, 1, 0, 16, 2, 64, [32, 0, 300], 16, 0),
    (1, 1, 0, 64, 8, 128, [1000], 64, 0),
    (2, 5, 0, 12, 4, 64, [100, 257], 16, 0),                      # three heads a K/V head
    (1, 5, 0, 7, 1, 128, [515], 0, 0),
    (2, 13, 4, 4, 2, 64, [65, 7], 0, 8),
    (1, 68, 4, 64, 8, 128, [700], 64, 16),
    (2, 68, 4, 4, 4, 128, [97, 0], 32, 33),                       # a prefix longer than a chunk
    (1, 100, 3, 32, 1, 64, [129], 0, 5),
    (1, 2, 1, 1, 1, 128, [640], 0, 1),
])
def test_against_float64(bits, n, R, masks, hq, hkv, hd, ctx, page, P):
    call, (out, tol), _ = case(n, R, masks, hq, hkv, hd, bits, ctx, page, P)
    near(call(), out, tol)


@BITS
def test_long_context_in_shares(bits):
    """A long key axis split over workgroups, lengths that leave some shares empty."""
    import paper_2401_12522_amd as bita
    assert bita.binding.tree_attention_mx_plan_info(3, 1, 8, 2, 128, bits, 9001)["splits"] > 8
    call, (out, tol), _ = case(3, 1, 0, 8, 2, 128, bits, [9001, 40, 0], 16)
    near(call(), out, tol)


def test_a_template_of_the_most_rows():
    import synth as s
    R = 512
    call, (out, tol), _ = case(1, R, 0, 2, 1, 64, 4, [50], seed=3)
    assert s is not None
    near(call(), out, tol)


@BITS
def test_hint_above_the_lengths_and_lengths_above_the_hint(bits):
    call, (out, tol), (cache, q, kr, vr, ck, cv, tmpl, seen, is_mask) = case(2, 3, 0, 4, 2, 128, bits, [70, 41], smax=200)
    import paper_2401_12522_amd as bita
    args = (tmpl, q.cuda(), cache, kr.cuda(), vr.cuda())
    near(bita.tree_attention_mx(*args, i32([70, 41]), 200), out, tol)
    out, tol = expected(q, ck, cv, kr, vr, [50, 41], seen, is_mask)           # read as at most the hint, and as 0 where negative
    near(bita.tree_attention_mx(*args, i32([70, 41]), 50), out, tol)
    out, tol = expected(q, ck, cv, kr, vr, [0, 41], seen, is_mask)
    near(bita.tree_attention_mx(*args, i32([-3, 41]), 60), out, tol)


@BITS
@pytest.mark.parametrize("ctx", [[60], [9000]])
def test_absent_rows_are_zero(bits, ctx):
    import paper_2401_12522_amd as bita
    call, (out, tol), _ = case(1, 12, 4, 4, 2, 64, bits, ctx, P=8)
    token = torch.arange(12, dtype=torch.int32)
    token[3], token[7], token[9] = -1, -1, -1                    # (row 9 is a mask row: its entry is no token)
    got = call(token=token.cuda()[None])
    out[0, [3, 7]], tol[0, [3, 7]] = 0, 0
    near(got, out, tol)
    assert bita is not None


@BITS
def test_what_no_row_sees_does_not_matter(bits):
    """Slots behind a length, rows on other branches and a prefix that token rows do not see hold NaN and infinities."""
    import paper_2401_12522_amd as bita
    n, R, hq, hkv, hd, P, ctx = 2, 9, 4, 2, 64, 8, [33, 50]
    call, (out, tol), (cache, q, kr, vr, ck, cv, tmpl, seen, is_mask) = case(n, R, 3, hq, hkv, hd, bits, ctx, 16, P, smax=80)
    bad = rows((n, hkv, 30, hd), 99, torch.bfloat16)
    bad[..., ::32] = float("nan")
    bita.kv_write_mx(cache, bad.cuda(), bad.cuda(), i32(ctx))
    # row j of the pass: NaN, +inf and -inf in V and K; only its descendants may notice
    j = 4
    kr2, vr2 = kr.clone(), vr.clone()
    kr2[:, :, j], vr2[:, :, j, 0::3], vr2[:, :, j, 1::3], vr2[:, :, j, 2::3] = float("nan"), float("nan"), float("inf"), float("-inf")
    pk, pv = rows((hkv, P, hd), 23, torch.bfloat16), rows((hkv, P, hd), 24, torch.bfloat16)
    pv[:, 2, 5], pk[:, 3, 1] = float("inf"), float("nan")
    got = bita.tree_attention_mx(tmpl, q.cuda(), cache, kr2.cuda(), vr2.cuda(), i32(ctx), 60, pk.cuda(), pv.cuda()).cpu().double().view(out.shape)
    blind = [r for r in range(R) if not seen[r, j] and not is_mask[r]]
    assert len(blind) > 2
    near(got[:, blind], out[:, blind], tol[:, blind])
    notice = [r for r in range(R) if seen[r, j] or is_mask[r]]
    assert got[:, notice].isnan().all(-1).all()                   # (a NaN score makes the whole row NaN)


@BITS
def test_infinite_values_that_are_seen(bits):
    """+inf, -inf and both in V of rows with finite scores: the sums are infinite or NaN where they have to be, finite elsewhere."""
    import paper_2401_12522_amd as bita
    call, (out, tol), (cache, q, kr, vr, ck, cv, tmpl, seen, is_mask) = case(1, 6, 0, 4, 2, 64, bits, [40], seed=2)
    vr2 = vr.clone()
    vr2[0, :, 0, 3], vr2[0, :, 0, 4], vr2[0, :, 0, 5], vr2[0, :, 0, 6] = float("inf"), float("-inf"), float("nan"), float("inf")
    vr2[0, :, 1, 6] = float("-inf")
    got = bita.tree_attention_mx(tmpl, q.cuda(), cache, kr.cuda(), vr2.cuda(), i32([40]), 40).cpu().double().view(out.shape)[0]
    for r in range(6):                                            # row 0 is everyone's ancestor
        assert (got[r, :, 3] == float("inf")).all() and (got[r, :, 4] == float("-inf")).all() and got[r, :, 5].isnan().all()
        assert got[r, :, 6].isnan().all() if seen[r, 1] else (got[r, :, 6] == float("inf")).all()
    keep = [c for c in range(64) if c not in (3, 4, 5, 6)]
    near(got[None][..., keep], out[..., keep], tol[..., keep])


@BITS
def test_a_cached_nan_reaches_its_own_sequence_and_block_only(bits):
    import paper_2401_12522_amd as bita
    call, (out, tol), (cache, q, kr, vr, ck, cv, tmpl, seen, is_mask) = case(2, 2, 0, 4, 2, 128, bits, [40, 45])
    one = rows((2, 2, 1, 128), 5, torch.bfloat16)
    v = one.clone()
    v[1, 1, 0, 70] = float("nan")
    bita.kv_write_mx(cache, one.cuda(), v.cuda(), i32([100, 44]))          # (the first sequence's is dropped)
    got = call().cpu().double().view(out.shape)
    assert got[1, :, 2:, 64:96].isnan().all()
    got[1, :, :, :] = out[1]
    near(got, out, tol)
    assert bita.tree_attention_mx(tmpl, q.cuda(), cache, kr.cuda(), vr.cuda(), i32([40, 44]), 45).isfinite().all()


@BITS
def test_large_scores_and_a_moving_maximum(bits):
    """Keys that grow along the axis, scores of several hundred: the running maximum moves in every chunk."""
    import paper_2401_12522_amd as bita
    n, hkv, hd, L = 1, 2, 64, 400
    cache = make(hkv, hd, n, L, bits)
    k = rows((n, hkv, L, hd), 1).mul(torch.linspace(0.1, 12, L)[:, None]).to(torch.bfloat16)
    v = rows((n, hkv, L, hd), 2, torch.bfloat16)
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), i32([0]))
    tmpl, seen, is_mask = template(3)
    q, kr, vr = rows((n, 3, 4, hd), 3).mul(3).to(torch.bfloat16), rows((n, hkv, 3, hd), 4, torch.bfloat16), rows((n, hkv, 3, hd), 5, torch.bfloat16)
    out, tol = expected(q, ref.rounded(k, bits), ref.rounded(v, bits), kr, vr, [L], seen, is_mask)
    near(bita.tree_attention_mx(tmpl, q.cuda(), cache, kr.cuda(), vr.cuda(), i32([L]), L), out, tol)


def test_rows_of_any_strides():
    """Pass rows as columns of one product, K and V with strides of their own."""
    import paper_2401_12522_amd as bita
    call, (out, tol), (cache, q, kr, vr, ck, cv, tmpl, seen, is_mask) = case(2, 5, 0, 4, 2, 64, 4, [40, 45])
    wide = torch.full((2, 5, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 4:6] = kr.cuda().transpose(1, 2)
    got = bita.tree_attention_mx(tmpl, q.cuda(), cache, wide[:, :, 4:6].transpose(1, 2), vr.cuda(), i32([40, 45]), 45)
    near(got, out, tol)


def test_far_slots_of_a_long_cache():
    """Codes beyond 2^32 bytes from the cache's start, one sequence's keys there."""
    import paper_2401_12522_amd as bita
    hkv, hd, smax = 8, 128, 8_500_000
    cache = bita.KVCacheMX(hkv, hd, 9, 1_000_000, bits=8)
    assert cache.k.numel() > 2 ** 32 and smax > 0
    tmpl, seen, is_mask = template(1)
    k, v = rows((1, hkv, 300, hd), 1, torch.bfloat16), rows((1, hkv, 300, hd), 2, torch.bfloat16)
    kk, vv = k.expand(9, -1, -1, -1).contiguous(), v.expand(9, -1, -1, -1).contiguous()
    bita.kv_write_mx(cache, kk.cuda(), vv.cuda(), i32([0] * 9))
    q, kr, vr = rows((9, 1, 16, hd), 3, torch.bfloat16), rows((9, hkv, 1, hd), 4, torch.bfloat16), rows((9, hkv, 1, hd), 5, torch.bfloat16)
    ctx = [0] * 8 + [300]
    out, tol = expected(q, ref.rounded(kk, 8), ref.rounded(vv, 8), kr, vr, ctx, seen, is_mask)
    near(bita.tree_attention_mx(tmpl, q.cuda(), cache, kr.cuda(), vr.cuda(), i32(ctx), 300), out, tol)


@BITS
def test_same_result_every_time_eager_and_replayed(bits):
    """Two captured calls with workspaces of their own, replayed between eager ones on new inputs."""
    import paper_2401_12522_amd as bita
    calls = [case(1, 1, 0, 8, 2, 128, bits, [3000], 16, seed=s)[2] for s in (1, 2)]
    held = []
    for cache, q, kr, vr, ck, cv, tmpl, seen, is_mask in calls:
        held.append((tmpl, q.cuda(), cache, kr.cuda(), vr.cuda(), i32([3000])))
    graphs, outs = [], []
    for a in held:
        ws = torch.empty(bita.lib().bita_tree_attention_mx_workspace_bytes(1, 1, 8, 2, 128, bits, 3000, 0), dtype=torch.uint8, device="cuda")
        out = torch.zeros((1, 1, 1024), dtype=torch.bfloat16, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            bita.tree_attention_mx(*a, 3000, out=out, workspace=ws)
        graphs.append(g)
        outs.append((out, ws))
    for turn in range(3):
        for a in held:
            a[1].copy_(rows(a[1].shape, 50 + turn, torch.bfloat16))
        for g in graphs:
            g.replay()
        want = [bita.tree_attention_mx(*a, 3000) for a in held]
        torch.cuda.synchronize()
        for (o, _), w in zip(outs, want):
            assert torch.equal(o, w)


RAGGED = [1500, 0, 1, 700, 64, 32, 33, 31, 900, 1499, 10, 128, 127, 129, 300, 256, 255]
CUTS = [
    (2, 20, 4, 2, 2, 64, [40, 33], 16, 5),
    (1, 35, 3, 4, 4, 128, [300], 64, 16),                         # three tiles a head that read the same keys
    (1, 1, 0, 2, 1, 64, [3000], 0, 40),
    (3, 1, 0, 2, 1, 128, [1500, 0, 31], 16, 0),                   # all shares but a few are one sequence's
    (17, 5, 2, 8, 2, 128, RAGGED, 64, 40),
    (70, 1, 0, 2, 1, 64, [(37 * i) % 1501 for i in range(70)], 16, 3),   # more sequences than a wave has lanes
    (8, 20, 2, 32, 16, 64, [40, 39, 31, 0, 1, 33, 32, 17], 32, 3),
    (1, 20, 2, 16, 16, 128, [1500], 0, 0),
    (1, 20, 0, 32, 32, 128, [3000], 0, 0),
    (17, 68, 4, 64, 2, 64, [40, 39, 31, 0, 1, 33, 32, 17, 40, 5, 6, 7, 8, 9, 10, 11, 12], 16, 3),
    (1, 130, 5, 16, 1, 128, [6000], 256, 16),
    (3, 130, 5, 16, 1, 128, [2000, 0, 900], 256, 70),
    (66, 16, 2, 16, 1, 64, [(211 * i) % 1801 for i in range(66)], 16, 3),
    (1, 512, 4, 2, 1, 64, [200], 0, 100),                         # the most rows, a prefix of two tiles
]


def cut_of(bits, n, R, masks, hq, hkv, hd, ctx, page, P):
    import paper_2401_12522_amd as bita
    plan = bita.binding.tree_attention_mx_plan_info(n, R, hq, hkv, hd, bits, max(ctx), P)
    return plan["queries"], plan["waves"], plan["splits"] > 1


def test_the_cases_below_are_cut_in_every_way():
    assert {cut_of(b, *c) for b in (4, 8) for c in CUTS} == {(q, w, s) for q, w in ((16, 4), (16, 8), (32, 4), (128, 4)) for s in (False, True)}


@BITS
@pytest.mark.parametrize("n,R,masks,hq,hkv,hd,ctx,page,P", CUTS)
def test_every_cut_of_a_launch(bits, n, R, masks, hq, hkv, hd, ctx, page, P):
    """The kinds of workgroups, with one share of the keys a sequence and with several, and a NaN among the pass' values, which reaches the rows that see it only."""
    call, (out, tol), (cache, q, kr, vr, _, _, tmpl, seen, _) = case(n, R, masks, hq, hkv, hd, bits, ctx, page, P, seed=7)
    near(call(), out, tol)
    at = R - masks - 1
    vr[:, :, at, 3] = float("nan")
    got = call().cpu().double().view(out.shape)
    assert torch.isnan(got[:, seen[:, at]][..., 3]).all()
    got[..., 3] = torch.where(seen[:, at][None, :, None], out[..., 3], got[..., 3])
    near(got, out, tol)


@BITS
@pytest.mark.parametrize("n,hint", [(1, 20000), (5, 20000), (70, 3000)])
def test_shares_are_cut_from_the_lengths_not_the_hint(bits, n, hint):
    """A launch for long sequences (as a captured graph holds it) over short ones, a few of them long, in turn: one workspace, another cut each time."""
    import paper_2401_12522_amd as bita
    tmpl, seen, is_mask = template(3)
    cache, ck, cv = filled(1, 64, n, 700, bits, 0, 5)
    cache = bita.KVCacheMX(1, 64, n, hint, bits=bits)
    k, v = rows((n, 1, 700, 64), 6, torch.bfloat16), rows((n, 1, 700, 64), 7, torch.bfloat16)
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), i32([0] * n))
    ck, cv = ref.rounded(k, bits), ref.rounded(v, bits)
    q, kr, vr = rows((n, 3, 2, 64), 1, torch.bfloat16), rows((n, 1, 3, 64), 2, torch.bfloat16), rows((n, 1, 3, 64), 3, torch.bfloat16)
    ws = torch.empty(bita.lib().bita_tree_attention_mx_workspace_bytes(n, 3, 2, 1, 64, bits, hint, 0), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    ctx = i32([0] * n)
    qc, kc, vc, out = q.cuda(), kr.cuda(), vr.cuda(), torch.empty((n, 3, 128), dtype=torch.bfloat16, device="cuda")
    call = lambda: bita.tree_attention_mx(tmpl, qc, cache, kc, vc, ctx, hint, out=out, workspace=ws)     # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for lengths in ([0] * n, [1] * (n - 1) + [700], [700] * n, [700] + [33] * (n - 1)):
        ctx.copy_(i32(lengths))
        want, tol = expected(q, ck, cv, kr, vr, lengths, seen, is_mask)
        for step in (g.replay, call):
            out.fill_(9.0)
            step()
            near(out, want, tol)


@BITS
@pytest.mark.parametrize("n,R,masks,hq,hkv,hd,ctx,page,P", CUTS)
def test_a_block_that_is_no_number_in_every_cut(bits, n, R, masks, hq, hkv, hd, ctx, page, P):
    """A cached V block with an infinity reads back as NaN: 32 columns of its sequence and K/V head, and nothing else."""
    import paper_2401_12522_amd as bita
    call, (out, tol), (cache, q, kr, vr, ck, cv, *_) = case(n, R, masks, hq, hkv, hd, bits, ctx, page, P, seed=9)
    b = max(range(n), key=lambda i: ctx[i])
    slot = ctx[b] // 2
    k, v = ck[:, :, slot: slot + 1].to(torch.bfloat16), cv[:, :, slot: slot + 1].to(torch.bfloat16)      # (what is there already, exact in bf16)
    v[b, 0, 0, 35] = float("inf")
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), i32([slot] * n), i32([int(i == b) for i in range(n)]))
    got = call().cpu().double().view(out.shape)
    group = hq // hkv
    assert torch.isnan(got[b, :, :group, 32:64]).all()
    got[b, :, :group, 32:64] = out[b, :, :group, 32:64]
    near(got, out, tol)


@BITS
@pytest.mark.parametrize("n,R,masks,hq,hkv,hd,ctx,page,P", [c for c in CUTS if c[1] > 4])
def test_absent_rows_in_every_cut(bits, n, R, masks, hq, hkv, hd, ctx, page, P):
    """Zeros for tree rows without a token, also where a NaN in their query would show; mask rows are never absent."""
    call, (out, tol), (cache, q, *_) = case(n, R, masks, hq, hkv, hd, bits, ctx, page, P, seed=11)
    token = torch.arange(n * R, dtype=torch.int32).view(n, R)
    gone = torch.zeros(n, R, dtype=torch.bool)
    gone[:, [1, 3, R - masks - 1]] = True
    gone[0, 2] = n > 1
    gone[:, R - masks:] = False
    token[gone] = -5
    token[:, R - masks:] = -1
    q[gone] = float("nan")
    got = call(token=token.cuda()).cpu().double().view(out.shape)
    assert (got[gone] == 0).all() and not torch.signbit(got[gone]).any()
    got[gone] = out[gone]
    near(got, out, tol)


def test_more_sequences_than_a_wave_has_lanes_in_wide_shares():
    """A large batch is cut by the hint: sequences with fewer shares than the longest, and with one."""
    n, R, ctx = 65, 16, [(53 * i) % 4001 for i in range(64)] + [4000]
    assert cut_of(8, n, R, 2, 8, 1, 64, ctx, 64, 3) == (128, 4, True)
    call, (out, tol), _ = case(n, R, 2, 8, 1, 64, 8, ctx, 64, 3, seed=13)
    got = call()
    near(got, out, tol)
    assert torch.equal(call(), got)
