"""Steps over the small cache from HIP graphs: norm with rotation, attention in every kind of workgroups, the write by a path, the way back (GPU)."""
import pytest
import torch

from test_gpu_kv_mx import i32, make, rows
from test_gpu_tree_attention_mx import template

pytestmark = pytest.mark.gpu

SIZES = [                                                         # sequences, rows, heads, K/V heads, head size, lengths, page, workgroup's queries and waves, split
    (1, 1, 8, 8, 128, [700], 64, (16, 8, False)),
    (2, 20, 2, 2, 64, [40, 33], 0, (16, 4, False)),
    (3, 1, 2, 1, 128, [1500, 0, 31], 16, (16, 8, True)),
    (8, 20, 32, 16, 64, [40, 39, 31, 0, 1, 33, 32, 17], 32, (32, 4, False)),
    (1, 130, 16, 1, 128, [6000], 256, (128, 4, True)),
]


class Step:
    """One layer's step of n sequences, every buffer its own but the workspace."""

    def __init__(self, n, R, hq, hkv, hd, ctx, page, seed, workspace=None):
        import paper_2401_12522_amd as bita
        self.bita, self.sizes, most = bita, (n, R, hq, hkv, hd), max(ctx) + 64
        self.tmpl = template(R, 0, seed)[0]
        self.cache = make(hkv, hd, n, most, 4, page, seed)
        fill = rows((n, hkv, max(max(ctx), 1), hd), seed + 1, torch.bfloat16).cuda()
        bita.kv_write_mx(self.cache, fill, fill, i32([0] * n))
        self.x, self.pos = rows((n * R, (hq + 2 * hkv) * hd), seed + 2, torch.float32).cuda(), i32([c + r for c in ctx for r in range(R)])
        angle = torch.arange(most + R, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(hd // 2, dtype=torch.float64) * 2 / hd)
        self.cos, self.sin = angle.cos().float().cuda(), angle.sin().float().cuda()
        self.gain = (1 + 0.2 * rows((hd,), seed + 3, torch.float32)).to(torch.bfloat16).cuda()
        self.ctx, self.hint = i32(ctx), max(ctx) + 32
        self.path, self.n_acc = i32([[0] * min(R, 3)] * n), i32([min(R, 3)] * n)
        e = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")     # noqa: E731
        self.q, self.k, self.v, self.out = e(n * R, hq, hd), e(n * R, hkv, hd), e(n * R, hkv, hd), e(n, R, hq * hd)
        self.back = e(n, hkv, min(R, 3), hd), e(n, hkv, min(R, 3), hd)
        self.ws = workspace

    def need(self):
        n, R, hq, hkv, hd = self.sizes
        return self.bita.lib().bita_tree_attention_mx_workspace_bytes(n, R, hq, hkv, hd, 4, self.hint, 0)

    def __call__(self):
        n, R, hq, hkv, hd = self.sizes
        self.bita.qk_norm_rope(self.x, self.pos, self.cos, self.sin, hq, hkv, self.gain, self.gain, q=self.q, k=self.k, v=self.v)
        k, v = (t.view(n, R, hkv, hd).transpose(1, 2) for t in (self.k, self.v))
        self.bita.tree_attention_mx(self.tmpl, self.q.view(n, R, hq, hd), self.cache, k, v, self.ctx, self.hint, out=self.out, workspace=self.ws)
        self.bita.kv_write_mx(self.cache, k, v, self.ctx, self.n_acc, self.path)
        self.bita.kv_read_mx(self.cache, *self.back, self.n_acc, start=self.ctx)

    def results(self):
        return [t.clone() for t in (self.out, *self.back, self.q, self.cache.k, self.cache.v_scale)]


def captured(step):
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    return g


@pytest.mark.parametrize("n,R,hq,hkv,hd,ctx,page,cut", SIZES)
def test_a_step_replayed(n, R, hq, hkv, hd, ctx, page, cut):
    """Inputs, lengths and cache change between the replays; each equals the calls made one by one, bit for bit."""
    import paper_2401_12522_amd as bita
    plan = bita.binding.tree_attention_mx_plan_info(n, R, hq, hkv, hd, 4, max(ctx) + 32, 0)
    assert (plan["queries"], plan["waves"], plan["splits"] > 1) == cut
    s = Step(n, R, hq, hkv, hd, ctx, page, 3)
    s.ws = torch.empty(max(s.need(), 16), dtype=torch.uint8, device="cuda")
    g = captured(s)
    for turn in range(3):
        s.x.copy_(rows(tuple(s.x.shape), 40 + turn, torch.float32))
        s.ctx.copy_(i32([c + turn if turn < 2 else min(c, 5) for c in ctx]))
        before = s.cache.k.clone(), s.cache.v.clone(), s.cache.k_scale.clone(), s.cache.v_scale.clone()
        s()
        want = s.results()
        for t, b in zip((s.cache.k, s.cache.v, s.cache.k_scale, s.cache.v_scale), before):
            t.copy_(b)
        for t in (s.out, *s.back, s.q):
            t.fill_(3.0)
        s.ws.fill_(255)
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(s.results(), want))


def test_graphs_that_share_a_workspace():
    """Two captured steps of different cuts over one workspace, one behind the other and in either order."""
    a, b = Step(3, 1, 2, 1, 128, [1500, 0, 31], 16, 3), Step(1, 130, 16, 1, 128, [6000], 256, 5)
    a.ws = b.ws = torch.empty(max(a.need(), b.need()), dtype=torch.uint8, device="cuda")
    want = []
    for s in (a, b):
        s()                                                     # (the rows that it writes are the same each time)
        want.append(s.results())
    ga, gb = captured(a), captured(b)
    for order in ((ga, gb), (gb, ga), (ga, gb, ga), (gb, gb, ga)):
        for s in (a, b):
            s.out.fill_(3.0)
        for g in order:
            g.replay()
        for s, w in ((a, want[0]), (b, want[1])):
            assert all(torch.equal(x, y) for x, y in zip(s.results(), w))


def test_prompt_attention_and_norm_replayed():
    import paper_2401_12522_amd as bita
    x = rows((300, (8 + 2 * 2) * 128), 1, torch.bfloat16).cuda()
    pos, cu = i32(list(range(300))), i32([0, 100, 100, 231, 290])
    angle = torch.arange(300, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)
    cos, sin = angle.cos().float().cuda(), angle.sin().float().cuda()
    q, k, out = (torch.zeros((300, w, 128), dtype=torch.bfloat16, device="cuda") for w in (8, 2, 8))
    out = out.view(300, 1024)

    def step():
        _, _, v = bita.qk_norm_rope(x, pos, cos, sin, 8, 2, q=q, k=k)
        bita.prompt_attention(q, k, v, cu, out=out)

    g = captured(step)
    for turn in range(3):
        x.copy_(rows(tuple(x.shape), 50 + turn, torch.bfloat16))
        cu.copy_(i32([[0, 100, 100, 231, 290], [3, 3, 4, 64, 300], [0, 0, 0, 0, 129]][turn]))
        out.fill_(2.0)
        step()
        want = out.clone()
        out.fill_(2.0)
        g.replay()
        assert torch.equal(out, want)
