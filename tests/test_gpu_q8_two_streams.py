"""8-bit calls on two streams at once (GPU): products whose k is split, and steps of one model, give what they give alone."""
import numpy as np
import pytest
import torch

import synth
from gpu_util import dev_i32
from test_gpu_q8_gemm import codes

pytestmark = pytest.mark.gpu


def _at_once(calls, turns=8):
    """Every call on a stream of its own, several times over; their last results."""
    streams, out = [torch.cuda.Stream() for _ in calls], [None] * len(calls)
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(turns):
        for i, call in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                out[i] = call()
    torch.cuda.synchronize()
    return out


def test_split_products():
    import paper_2401_12522_amd as bita
    calls = []
    for m, n, k, seed in ((68, 4096, 11008, 1), (300, 1024, 9001, 3), (5, 256, 8192, 5)):
        assert bita.binding.gemm_q8_plan_info(m, n, k)["splits"] > 1
        (a, sa), (w, sw) = codes(m, k, seed), codes(n, k, seed + 1)
        packed = bita.pack_weight_q8(w)
        calls.append(lambda a=a, sa=sa, p=packed, sw=sw, n=n: bita.gemm_q8(a, sa, p, sw, n))
    alone = [c().clone() for c in calls]
    for y, want in zip(_at_once(calls), alone):
        assert torch.equal(y, want)


def test_steps_of_one_model():
    import paper_2401_12522_amd as bita
    cfg = synth.get_config("tiny_gqa", d_model=256, n_heads=128, n_kv_heads=64, d_ffn=8192)      # (split products in every layer)
    model = bita.Model(cfg, synth.SynthWeights(cfg, seed=0, norm_std=0.3, prefix_std=1.0), max_pos=320, int8=True)
    tin = synth.attach_mask_groups(synth.random_tree(12, 3, 1), [0], cfg.n_mask)
    tmpl = bita.TreeTemplate(tin.parent, tin.is_mask, tin.n_tree, cfg.n_mask)
    calls, bufs = [], []
    for i, ctx in enumerate((60, 17)):
        g = torch.Generator(device="cuda").manual_seed(i)
        kv = bita.KVState(cfg, cfg.n_layers, 1, 256, tmpl.rows)
        kv.k_cache.copy_(0.3 * torch.randn(kv.k_cache.shape, device="cuda", generator=g))
        kv.v_cache.copy_(0.3 * torch.randn(kv.v_cache.shape, device="cuda", generator=g))
        buf, start = bita.StepBuffers(model, tmpl, 1, tmpl.kmax, want_logits=True), dev_i32([ctx])
        root, cand = dev_i32([i + 3]), dev_i32(np.random.default_rng(i).integers(0, cfg.vocab, size=(1, cfg.n_mask, tmpl.kmax)))

        def call(kv=kv, buf=buf, start=start, root=root, cand=cand, ctx=ctx):
            kv.ctx_len.copy_(start)
            bita.decode_step(model, kv, ctx, tmpl, buf, 1, root, cand)
            return buf.logits
        calls.append(call)
        bufs.append(buf)
    alone = []
    for call, buf in zip(calls, bufs):
        call()
        torch.cuda.synchronize()
        alone.append((buf.logits.clone(), buf.emitted.clone(), buf.bonus.clone()))
    _at_once(calls)
    for buf, (logits, emitted, bonus) in zip(bufs, alone):
        assert torch.equal(buf.logits, logits) and torch.equal(buf.bonus, bonus) and torch.equal(buf.emitted, emitted)
