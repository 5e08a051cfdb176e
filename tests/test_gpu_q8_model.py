"""The 8-bit operators together (GPU): a layer's feed-forward part from the calls themselves, eager and replayed, and whole passes of
a model whose layers are 8-bit against a float64 pass with the same integers.

How far logits may be off: both sides round the same rows to the same integers until the sides' own rounding (attention and
rotation, about 1e-5 of a row) takes one value across a border, a whole step of a / 127 away.  That changes the next rows by some
1e-3, which takes 127 * 1e-3, an eighth, of their values across a border, each by a step: sqrt(1/8) steps root mean square against the
0.29 of rounding itself.  From there on the two sides' rounding errors are as good as independent, and differ by sqrt(2) of one side's,
the distance of the 8-bit reference from the unrounded pass: 1.5 of it is allowed root mean square, six times that anywhere (a few
ten thousand values of a normal distribution stay within 4.5).  A product with a wrong scale, row or column is off by the logits' own size,
60 times that distance.  Rows where no value has crossed a border agree to fp32; the stages are checked one by one in the first test.

The rule had been 0.25 of that distance, from the first crossing alone without those that follow from it.
"""
import numpy as np
import pytest
import torch

import oracle
import synth
from gpu_util import dev_i32, load_cache, read_cache
from oracle.decode import prefill as oracle_prefill
from oracle.tree import ancestors_or_self, build_tree_tokens, derive_template
from q8_reference import forward_rows_q8
from test_gpu_q8_gemm import check as check_product
from test_gpu_q8_rows import check as check_rows

pytestmark = pytest.mark.gpu


def _weight(n, k, seed):
    import paper_2401_12522_amd as bita
    g = torch.Generator(device="cuda").manual_seed(seed)
    return bita.quantize_rows((torch.randn(n, k, device="cuda", generator=g) * 0.05).to(torch.bfloat16))


@pytest.mark.parametrize("m,d,f", [(1, 256, 688), (5, 512, 1376), (68, 1024, 2752), (171, 520, 1392), (700, 1024, 1376)])
def test_feed_forward_of_a_layer(m, d, f):
    """x += delta; y = FFN(norm(x)); then the next norm adds y.  Every stage against its definition on what it was given."""
    import paper_2401_12522_amd as bita
    (wg, sg), (wu, su), (wd, sd) = _weight(f, d, 1), _weight(f, d, 2), _weight(d, f, 3)
    gu = torch.empty(bita.packed_q8_bytes(2 * f, d), dtype=torch.uint8, device="cuda")
    bita.pack_weight_q8(wg, gu, 0, 2, total_rows=2 * f)
    bita.pack_weight_q8(wu, gu, 1, 2, total_rows=2 * f)
    s_gu = torch.stack([sg.view(-1, 16), su.view(-1, 16)], 1).reshape(-1)
    w_gu = torch.stack([wg.reshape(-1, 16, d), wu.reshape(-1, 16, d)], 1).reshape(2 * f, d)
    down = bita.pack_weight_q8(wd)
    g = torch.Generator(device="cuda").manual_seed(4)
    x0, delta0 = torch.randn(m, d, device="cuda", generator=g), 0.3 * torch.randn(m, d, device="cuda", generator=g)
    x0[m // 2], delta0[m // 2] = 0, 0                                    # a row that is absent
    gain = (1 + 0.2 * torch.randn(d, device="cuda", generator=g)).to(torch.bfloat16)
    x, delta = x0.clone(), delta0.clone()

    def layer():
        out = {}
        out["h"] = bita.norm_q8(x, gain, 1e-5, delta=delta)
        out["gu"] = bita.gemm_q8(*out["h"], gu, s_gu, 2 * f)
        out["act"] = bita.silu_mul_q8(out["gu"], tile=16)
        out["y"] = bita.gemm_q8(*out["act"], down, sd, d)
        out["next"] = bita.norm_q8(x, gain, 1e-5, delta=out["y"], total=torch.empty_like(x))
        return out

    def reset():
        x.copy_(x0)
        delta.copy_(delta0)

    eager = layer()
    h = x0 + delta0
    assert torch.equal(x, h)
    factor = lambda t: 1 / torch.sqrt(t.double().square().mean(1) + 1e-5)                      # noqa: E731
    check_rows(*eager["h"], h.double() * gain.double(), factor(h))
    check_product(eager["gu"], *eager["h"], w_gu, s_gu)
    gate, up = eager["gu"].view(m, -1, 2, 16).unbind(2)
    gate, up = gate.reshape(m, f).double(), up.reshape(m, f).double()
    check_rows(*eager["act"], gate / (1 + torch.exp(-gate)) * up)
    check_product(eager["y"], *eager["act"], wd, sd)
    check_rows(*eager["next"], (h + eager["y"]).double() * gain.double(), factor(h + eager["y"]))
    assert not eager["y"][m // 2].any()
    # replayed, with the program's own work between the replays
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        captured = layer()
    for _ in range(3):
        reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, h)
        for name, value in eager.items():
            for a, b in zip(value if isinstance(value, tuple) else (value,), captured[name] if isinstance(value, tuple) else (captured[name],)):
                assert torch.equal(a, b), name
        bita.quantize_rows(torch.randn(50, 300, device="cuda"))


def _model(cfg_name, smax=256, **more):
    import paper_2401_12522_amd as bita
    cfg = synth.get_config(cfg_name)
    w = synth.SynthWeights(cfg, seed=0, norm_std=0.3, prefix_std=1.0)
    return cfg, oracle.OracleModel(cfg, w), bita.Model(cfg, w, max_pos=smax + 64, int8=True, **more)


@pytest.mark.parametrize("cfg_name", ["tiny", "tiny_gqa"])
@pytest.mark.parametrize("rows,ctx,page", [(8, 33, 0), (1, 1, 0), (40, 100, 0), (8, 70, 16)])
def test_pass_of_an_8_bit_model(cfg_name, rows, ctx, page):
    import paper_2401_12522_amd as bita
    cfg, om, model = _model(cfg_name)
    tin = synth.attach_mask_groups(synth.random_tree(rows, 3, 0) if rows > 1 else [-1], [0], cfg.n_mask)
    d = derive_template(tin.parent, tin.is_mask, cfg.n_mask)
    tokens_ctx = synth.random_context(cfg.vocab, ctx + 1, 0)
    ck, cv = oracle_prefill(om, tokens_ctx)
    ck, cv = [synth.bf16_round(a) for a in ck], [synth.bf16_round(a) for a in cv]
    cand = np.random.default_rng(0).integers(0, cfg.vocab, size=(cfg.n_mask, max(d.kmax, 1))).astype(np.int32)
    tokens = build_tree_tokens(d, int(tokens_ctx[-1]), cand, 0, 0)
    pos, vis = [ctx + d.depth[r] for r in range(d.R)], [ancestors_or_self(d.parent, r) for r in range(d.R)]
    want, k_ref, v_ref = forward_rows_q8(om, tokens, d.is_mask, d.mask_index, pos, vis, ck, cv)
    plain, k_plain, _ = oracle.forward_rows(om, tokens, d.is_mask, d.mask_index, pos, vis, ck, cv)
    tmpl = bita.TreeTemplate(tin.parent, tin.is_mask, tin.n_tree, cfg.n_mask)
    if page:
        kv = bita.PagedKVState(cfg, cfg.n_layers, 1, 256, tmpl.rows, page)
        kv.load_contiguous(0, torch.tensor(np.stack(ck)).permute(0, 2, 1, 3).to(torch.bfloat16).cuda(), torch.tensor(np.stack(cv)).permute(0, 2, 1, 3).to(torch.bfloat16).cuda(), ctx)
    else:
        kv = bita.KVState(cfg, cfg.n_layers, 1, 256, tmpl.rows)
        load_cache(kv, ck, cv)
    buf = bita.StepBuffers(model, tmpl, 1, max(d.kmax, 1), want_logits=True)
    bita.decode_step(model, kv, ctx, tmpl, buf, 1, dev_i32([int(tokens_ctx[-1])]), dev_i32(cand[None]))
    torch.cuda.synchronize()
    got = buf.logits[0].double().cpu().numpy()
    assert buf.token[0].cpu().tolist() == tokens
    live = np.array([bool(d.is_mask[r]) or tokens[r] >= 0 for r in range(d.R)])
    off, rounding = got[live] - want[live], want[live] - plain[live]
    def near(off, rounding):
        allowed = 1.5 * np.sqrt((rounding ** 2).mean())
        assert np.sqrt((off ** 2).mean()) <= allowed and np.abs(off).max() <= 6 * allowed

    assert np.isfinite(got).all()
    near(off, rounding)
    assert not got[~live].any()
    for l in range(cfg.n_layers):                                          # the rows' keys and values, before the commit rounds nothing more
        k = kv.k_tree[l, 0].permute(1, 0, 2).double().cpu().numpy()
        near(k[live] - k_ref[l][live], k_ref[l][live] - k_plain[l][live])


@pytest.mark.parametrize("rows,ctx", [(8, 33), (1, 1), (40, 100)])
def test_pass_whose_products_are_split(rows, ctx, monkeypatch):
    """The output and down projections' k is split: the norms behind them, and at the end the LM head's, take up the sums."""
    import paper_2401_12522_amd as bita
    cfg = synth.get_config("tiny", d_model=256, n_heads=128, n_kv_heads=128, d_ffn=8192, n_layers=2)
    monkeypatch.setitem(synth.configs.CONFIGS, "long sums", cfg)
    for k in (cfg.n_heads * cfg.head_dim, cfg.d_ffn):
        assert bita.binding.gemm_q8_plan_info(rows + cfg.n_mask, cfg.d_model, k)["splits"] > 1
    test_pass_of_an_8_bit_model("long sums", rows, ctx, 0)


def _greedy(model, cfg, tokens, n, tree):
    """Tokens and smallest top-2 distance of a free-running decode from a prefilled context."""
    import paper_2401_12522_amd as bita
    tin = synth.attach_mask_groups(tree, [0], cfg.n_mask)
    tmpl = bita.TreeTemplate(tin.parent, tin.is_mask, tin.n_tree, cfg.n_mask)
    kv = bita.KVState(cfg, cfg.n_layers, 1, 256, max(tmpl.rows, 16))
    toks = dev_i32(tokens[None])
    root = bita.prefill(model, kv, 0, toks, 16)
    kv.resize_rows(cfg.n_layers, cfg, tmpl.rows)
    kmax = max(tmpl.kmax, 1)
    buf = bita.StepBuffers(model, tmpl, 1, kmax, want_logits=True)
    cand = torch.full((1, cfg.n_mask, kmax), -1, dtype=torch.int32, device="cuda")
    group, shift = dev_i32([0]), dev_i32([cfg.n_mask])
    out, gaps, ctx = [int(root)], [], len(tokens)
    while len(out) < n:
        bita.decode_step(model, kv, ctx, tmpl, buf, 1, root, cand, group, shift)
        acc = int(buf.n_acc[0])
        out += buf.emitted[0, :acc].cpu().tolist()
        for r in buf.path[0, :acc].cpu().tolist():
            top = buf.logits[0, r].topk(2).values
            gaps.append(float(top[0] - top[1]))
        root, cand, group, shift = buf.bonus.clone(), buf.topk_ids.clone(), buf.next_group.clone(), buf.next_shift.clone()
        ctx += acc
    return out[:n], gaps[: n - 1]


@pytest.mark.parametrize("cfg_name", ["tiny", "tiny_gqa"])
def test_drafting_changes_no_token(cfg_name):
    """Drafted decoding of the 8-bit model gives the tokens of one-row decoding, up to the first that another rounding of attention could change."""
    cfg, om, model = _model(cfg_name)
    tokens = synth.random_context(cfg.vocab, 37, 3)
    one, gaps = _greedy(model, cfg, tokens, 24, [-1])
    drafted, _ = _greedy(model, cfg, tokens, 24, synth.full_branching_tree([4, 3, 2, 1], 24))
    sure = 1 + next((i for i, g in enumerate(gaps) if g < 1e-2), len(gaps))
    assert sure >= 2 and drafted[:sure] == one[:sure]


def test_prefill_of_an_8_bit_model_is_its_passes():
    """Chunked prefill, ragged lengths and all: the cache and the next tokens of one-row passes over the same context."""
    import paper_2401_12522_amd as bita
    cfg, om, model = _model("tiny")
    lens = [29, 1, 16]
    toks = np.stack([synth.random_context(cfg.vocab, 29, s) for s in range(3)])
    kv = bita.KVState(cfg, cfg.n_layers, 3, 64, 16)
    nxt = bita.prefill(model, kv, 0, dev_i32(toks), 16, seq_len=dev_i32(lens)).cpu().tolist()
    assert kv.ctx_len.cpu().tolist() == lens
    one = bita.TreeTemplate([-1], [0], 1, 0)
    for b, n in enumerate(lens):
        single = bita.KVState(cfg, cfg.n_layers, 1, 64, 1)
        buf = bita.StepBuffers(model, one, 1, 1, want_logits=True)
        for i in range(n):
            bita.decode_step(model, single, i, one, buf, 1, dev_i32([int(toks[b, i])]), None)
        top = buf.logits[0, 0].topk(2)
        if float(top.values[0] - top.values[1]) > 1e-2:
            assert nxt[b] == int(buf.bonus[0])
        plain = oracle_prefill(om, np.append(toks[b, :n], 0))
        for got, want, exact in zip(read_cache(kv, b), read_cache(single, 0), plain):
            for l in range(cfg.n_layers):
                allowed = 1.5 * np.sqrt(((want[l] - exact[l]) ** 2).mean())
                assert np.sqrt(((got[l] - want[l]) ** 2).mean()) <= allowed and np.abs(got[l] - want[l]).max() <= 6 * allowed
