"""Whole steps of a model with 8-bit layers (GPU): several sequences of unequal lengths, a step in a graph, and a layer of real widths,
against a float64 pass with the same integers.

Two rules.  Logits and later layers: within 1.5 times the distance that the 8-bit rounding itself makes (root mean square, six times that anywhere):
once a value has crossed a rounding border the two sides' rounding errors are independent of each other.  The first layer's keys and values: no border can be
crossed in front of them, for the rows are embeddings, and they are the exact value but for its rounding to bf16 (2^-8 of it) and the roundings in
fp32 before that: three of a product of scales, and for keys the rotation's two products, sum and table, each half a step of a value no larger
than twice the row's largest: 16 * 2^-24 of that in all.  There the integers are those of embedding times gain, which doubles hold: a row's factor, divided out
first as the pass does it, moves values that lie on a border off it."""
import numpy as np
import pytest
import torch

import oracle
import synth
from gpu_util import dev_i32, load_cache
from oracle.tree import ancestors_or_self, build_tree_tokens, derive_template
from oracle.model import rope_rotate
from q8_reference import forward_rows_q8, rows_q8

pytestmark = pytest.mark.gpu


def _near(off, rounding):
    allowed = 1.5 * np.sqrt((rounding ** 2).mean())
    assert np.sqrt((off ** 2).mean()) <= allowed and np.abs(off).max() <= 6 * allowed


def _rounded_once(got, want):
    slack = 16 * 2.0 ** -24 * np.abs(want).max(axis=-1, keepdims=True)
    assert bool((np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + slack).all())


def _first_layer(cfg, om, d, tokens, pos):
    """Keys and values of the first layer, from its rows' exact integers."""
    x = np.zeros((d.R, cfg.d_model))
    for r in range(d.R):
        if d.is_mask[r]:
            x[r] = om.w("mask_emb")[d.mask_index[r]]
        elif tokens[r] >= 0:
            x[r] = om.w("tok_emb")[tokens[r]]
    v = x * om.w("attn_norm", 0)
    q, s = rows_q8(v)[0], np.abs(v).max(1) / 127 / np.sqrt((x * x).mean(1) + cfg.rms_eps)
    out = []
    for name in ("wk", "wv"):
        qw, sw = rows_q8(om.w(name, 0))
        out.append(((q @ qw.T) * s[:, None] * sw).reshape(d.R, cfg.n_kv_heads, cfg.head_dim))
    return np.stack([rope_rotate(out[0][r], pos[r], cfg.rope_theta) for r in range(d.R)]), out[1]


def _cache(cfg, ctx, seed):
    """Keys and values of a context, bf16 numbers of the size that the layers give."""
    g = np.random.default_rng(seed)
    draw = lambda: [synth.bf16_round(0.3 * g.standard_normal((ctx, cfg.n_kv_heads, cfg.head_dim))) for _ in range(cfg.n_layers)]     # noqa: E731
    return draw(), draw()


def _check_sequence(cfg, om, d, tokens, ctx, ck, cv, logits, k_tree, v_tree):
    pos, vis = [ctx + d.depth[r] for r in range(d.R)], [ancestors_or_self(d.parent, r) for r in range(d.R)]
    want, k_ref, v_ref = forward_rows_q8(om, tokens, d.is_mask, d.mask_index, pos, vis, ck, cv)
    plain, k_plain, v_plain = oracle.forward_rows(om, tokens, d.is_mask, d.mask_index, pos, vis, ck, cv)
    live = np.array([bool(d.is_mask[r]) or tokens[r] >= 0 for r in range(d.R)])
    assert np.isfinite(logits).all() and not logits[~live].any()
    _near(logits[live] - want[live], want[live] - plain[live])
    for l in range(cfg.n_layers):
        for got, ref, exact in ((k_tree[l], k_ref[l], k_plain[l]), (v_tree[l], v_ref[l], v_plain[l])):
            _near(got[live] - ref[live], ref[live] - exact[live])
            assert not got[~live].any()
    for got, ref in zip((k_tree[0], v_tree[0]), _first_layer(cfg, om, d, tokens, pos)):
        _rounded_once(got[live], ref[live])


def _rows(t):
    """[L][Hkv][R][hd] of a sequence -> [L][R][Hkv][hd] doubles."""
    return t.permute(0, 2, 1, 3).double().cpu().numpy()


def _step(cfg, w, model, tin, lens, smax, absent, seed):
    """One step of len(lens) sequences: (buffers, kv, the call, tokens, caches, d)."""
    import paper_2401_12522_amd as bita
    B, d = len(lens), derive_template(tin.parent, tin.is_mask, cfg.n_mask)
    tmpl = bita.TreeTemplate(tin.parent, tin.is_mask, tin.n_tree, cfg.n_mask)
    kv = bita.KVState(cfg, cfg.n_layers, B, smax, tmpl.rows)
    caches = [_cache(cfg, n, seed + b) for b, n in enumerate(lens)]
    for b, (ck, cv) in enumerate(caches):
        load_cache(kv, ck, cv, b=b)
    roots = synth.random_context(cfg.vocab, B, seed)
    cand = np.random.default_rng(seed).integers(0, cfg.vocab, size=(B, cfg.n_mask, max(d.kmax, 1))).astype(np.int32)
    for b, level, rank in absent:
        cand[b, level, rank:] = -1
    tokens = [build_tree_tokens(d, int(roots[b]), cand[b], 0, 0) for b in range(B)]
    buf = bita.StepBuffers(model, tmpl, B, max(d.kmax, 1), want_logits=True)
    args = (dev_i32(roots), dev_i32(cand))
    call = lambda: bita.decode_step(model, kv, max(lens), tmpl, buf, B, *args)      # noqa: E731
    return buf, kv, call, tokens, caches, d


@pytest.mark.parametrize("cfg_name", ["tiny", "tiny_gqa"])
@pytest.mark.parametrize("lens,rows", [([70, 33, 1], 8), ([5, 120], 24), ([1, 2, 3, 64, 65, 100, 17], 5)])
def test_sequences_of_unequal_lengths(cfg_name, lens, rows):
    import paper_2401_12522_amd as bita
    cfg = synth.get_config(cfg_name)
    w = synth.SynthWeights(cfg, seed=0, norm_std=0.3, prefix_std=1.0)
    om, model = oracle.OracleModel(cfg, w), bita.Model(cfg, w, max_pos=320, int8=True)
    tin = synth.attach_mask_groups(synth.random_tree(rows, 3, 1), [0], cfg.n_mask)
    buf, kv, call, tokens, caches, d = _step(cfg, w, model, tin, lens, 256, [(0, 0, 1)], 11)
    call()
    torch.cuda.synchronize()
    assert buf.token.cpu().tolist() == tokens and any(t < 0 for t in tokens[0])
    for b, n in enumerate(lens):
        _check_sequence(cfg, om, d, tokens[b], n, *caches[b], buf.logits[b].double().cpu().numpy(), _rows(kv.k_tree[:, b]), _rows(kv.v_tree[:, b]))


@pytest.mark.parametrize("name,lens,absent", [("7b", [45], []), ("7b", [20, 90], [(0, 1, 2), (1, 0, 3)]), ("70b", [30], [(0, 2, 0)])])
def test_a_layer_of_real_widths(name, lens, absent):
    """64-node trees with their mask rows; the 70B shape with a quarter of its feed-forward width, for the float64 passes' sake."""
    import paper_2401_12522_amd as bita
    cfg = synth.get_config(name, n_layers=1, vocab=2048, **({"d_ffn": 7168} if name == "70b" else {}))
    w = synth.SynthWeights(cfg, seed=1, device="cuda", norm_std=0.3, prefix_std=1.0)
    model = bita.Model(cfg, w, max_pos=320, int8=True)
    tin = synth.attach_mask_groups(synth.full_branching_tree([4, 3, 2, 1], 64), [0], cfg.n_mask)
    buf, kv, call, tokens, caches, d = _step(cfg, w, model, tin, lens, 256, absent, 7)
    call()
    torch.cuda.synchronize()
    assert buf.token.cpu().tolist() == tokens
    om = oracle.OracleModel(cfg, w)
    for b, n in enumerate(lens):
        _check_sequence(cfg, om, d, tokens[b], n, *caches[b], buf.logits[b].double().cpu().numpy(), _rows(kv.k_tree[:, b]), _rows(kv.v_tree[:, b]))


@pytest.mark.parametrize("cfg_name,lens", [("tiny_gqa", [40]), ("tiny", [17, 64, 3])])
def test_a_step_in_a_graph(cfg_name, lens):
    """Captured and replayed, with other eager work and synchronizations between the replays: every output as the eager step's."""
    import paper_2401_12522_amd as bita
    cfg = synth.get_config(cfg_name)
    w = synth.SynthWeights(cfg, seed=0, norm_std=0.3, prefix_std=1.0)
    model = bita.Model(cfg, w, max_pos=320, int8=True)
    tin = synth.attach_mask_groups(synth.random_tree(12, 3, 1), [0], cfg.n_mask)
    buf, kv, call, tokens, caches, d = _step(cfg, w, model, tin, lens, 256, [(0, 0, 1)], 5)
    names = ("token", "argmax", "topk_ids", "topk_val", "logits", "path", "n_acc", "bonus", "emitted", "next_group", "next_shift")
    state = lambda: {n: getattr(buf, n).clone() for n in names} | {n: getattr(kv, n).clone() for n in ("k_cache", "v_cache", "k_tree", "v_tree", "ctx_len")}     # noqa: E731
    start, k0, v0 = kv.ctx_len.clone(), kv.k_cache.clone(), kv.v_cache.clone()

    def reset():
        kv.ctx_len.copy_(start)
        kv.k_cache.copy_(k0)
        kv.v_cache.copy_(v0)
        for n in names:
            getattr(buf, n).fill_(-7)

    reset()
    call()
    torch.cuda.synchronize()
    eager = state()
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in state().items():
            assert torch.equal(t, eager[n]), n
        bita.quantize_rows(torch.randn(50, 300, device="cuda"))
        torch.cuda.synchronize()
