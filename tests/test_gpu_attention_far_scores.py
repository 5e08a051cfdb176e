"""Attention over the small cache and over prompts (GPU) where scores are so far apart that fp32 has no digits behind the point for them: the largest takes all, by
whatever kernel."""
import math

import pytest
import torch

import mx_reference as ref
from test_gpu_kv_mx import i32, make, rows
from test_gpu_prompt_attention import starts
from test_gpu_tree_attention_mx import BITS, cut_of, template

pytestmark = pytest.mark.gpu
SIZES = pytest.mark.parametrize("exponent", [12, 16, 20, 30])      # of q and of k


def check(got, q, k, v, seen):
    """got [n][hd] of queries q [n][hd] over k, v [m][hd]: the value of the largest score, where fp32 (a product of hd terms, its scaling: (hd + 7) units of 2^-24 of
    the sum of magnitudes, for each of two scores) tells it from the next by more than 40 nats, of which 2^18 keys leave nothing.  Returns how many are told apart."""
    q, k, v, got = (t.double() for t in (q, k, v, got))
    hd = q.shape[-1]
    s = (q @ k.T / math.sqrt(hd)).masked_fill(~seen, -math.inf)
    size = (q.abs() @ k.abs().T / math.sqrt(hd)).masked_fill(~seen, 0.0).amax(-1)
    top, at = s.topk(2, -1) if s.shape[1] > 1 else (torch.cat([s, s - math.inf], -1), torch.zeros(len(s), 2, dtype=torch.long))
    apart = top[:, 0] - top[:, 1] > 40 + 2 * (hd + 7) * 2.0 ** -24 * size
    want = v[at[:, 0]]
    assert got.isfinite().all()
    assert ((got - want).abs()[apart] <= ref.HALF_BF16 * want.abs()[apart]).all()
    return int(apart.sum()), len(apart)


def scaled(shape, seed, exponent):
    return (rows(shape, seed).clamp(-4, 4) * 2.0 ** exponent).to(torch.bfloat16)


@BITS
@SIZES
@pytest.mark.parametrize("n,R,hq,hkv,hd,L,cut", [
    (1, 1, 8, 2, 128, 330, (16, False)), (8, 20, 32, 16, 64, 330, (32, False)), (17, 68, 64, 2, 64, 330, (128, False)), (9, 68, 64, 4, 128, 330, (128, False)),
    (1, 130, 16, 1, 128, 6000, (128, True)), (1, 1, 2, 1, 64, 3000, (16, True))])
def test_over_the_cache(bits, exponent, n, R, hq, hkv, hd, L, cut):
    import paper_2401_12522_amd as bita
    queries, _, split = cut_of(bits, n, R, 0, hq, hkv, hd, [L], 0, 0)
    assert (queries, split) == cut
    tmpl, seen, _ = template(R)
    q, k, v = scaled((1, R, hq, hd), 81, exponent), scaled((1, hkv, L, hd), 82, exponent), rows((1, hkv, L, hd), 83, torch.bfloat16)
    kr, vr = scaled((1, hkv, R, hd), 84, exponent), rows((1, hkv, R, hd), 85, torch.bfloat16)
    cache = make(hkv, hd, n, L, bits)
    up = lambda t: t.expand(n, -1, -1, -1).contiguous().cuda()      # noqa: E731  (the sequences are alike)
    bita.kv_write_mx(cache, up(k), up(v), i32([0] * n))
    got = bita.tree_attention_mx(tmpl, up(q), cache, up(kr), up(vr), i32([L] * n), L)
    assert torch.equal(got, got[:1].expand_as(got))
    got = got[0].cpu().view(R, hq, hd)
    told = of = 0
    for h in range(hq):
        g = h // (hq // hkv)
        a, b = check(got[:, h], q[0, :, h], torch.cat([ref.rounded(k[0, g], bits), kr[0, g].double()]), torch.cat([ref.rounded(v[0, g], bits), vr[0, g].double()]),
                     torch.cat([torch.ones(R, L, dtype=torch.bool), seen], 1))
        told, of = told + a, of + b
    assert told > 0.8 * of


@SIZES
@pytest.mark.parametrize("hd", [64, 128])
def test_over_prompts(hd, exponent):
    import paper_2401_12522_amd as bita
    lens, hq, hkv = [90, 300], 4, 2
    cu = starts(lens)
    q, k, v = scaled((cu[-1], hq, hd), 91, exponent), scaled((cu[-1], hkv, hd), 92, exponent), rows((cu[-1], hkv, hd), 93, torch.bfloat16)
    got = bita.prompt_attention(q.cuda(), k.cuda(), v.cuda(), i32(cu)).cpu().view(cu[-1], hq, hd)
    told = of = 0
    for a, b in zip(cu, cu[1:]):
        for h in range(hq):
            g = h // (hq // hkv)
            x, y = check(got[a:b, h], q[a:b, h], k[a:b, g], v[a:b, g], torch.ones(b - a, b - a, dtype=torch.bool).tril())
            told, of = told + x, of + y
    assert told > 0.8 * of
