"""Attention over the small cache and over prompts (GPU) where the first keys' scores are minus infinity in fp32 (q and k so far apart that they overflow): those
keys have no weight, and what the keys behind them give must not depend on them."""
import math

import pytest
import torch

import mx_reference as ref
from test_gpu_kv_mx import i32, make, rows
from test_gpu_prompt_attention import expected as expected_of_prompts
from test_gpu_tree_attention_mx import BITS, cut_of, expected, near, template

pytestmark = pytest.mark.gpu
FAR = 64                                                          # keys without weight: a tile


def queries_and_keys(q_shape, k_shape, seed, peaks={}):
    """Scores of ordinary size and, in octaves, `peaks` {slot: score}; minus infinity for the first keys and queries whose first value is not 0."""
    hd = q_shape[-1]
    side = torch.where(rows((hd,), seed) > 0, 1.0, -1.0)
    q = side + 0.3 * rows(q_shape, seed + 1).clamp(-1, 1)
    k = 0.1 * rows(k_shape, seed + 2).clamp(-1, 1)
    for slot, octaves in peaks.items():
        k[..., slot, :] = side * octaves * math.log(2) / math.sqrt(hd)
    q[..., 0], k[..., 0], k[..., :FAR, 0] = 2.0 ** 70, 0.0, -2.0 ** 80
    return q.to(torch.bfloat16), k.to(torch.bfloat16)


@BITS
@pytest.mark.parametrize("n,R,hq,hkv,hd,L,cut", [
    (1, 1, 8, 2, 128, 330, (16, False)), (8, 20, 32, 16, 64, 330, (32, False)), (17, 68, 64, 2, 64, 330, (128, False)), (9, 68, 64, 4, 128, 330, (128, False)),
    (1, 130, 16, 1, 128, 6000, (128, True)), (1, 1, 2, 1, 64, 3000, (16, True))])
def test_over_the_cache(bits, n, R, hq, hkv, hd, L, cut):
    import paper_2401_12522_amd as bita
    queries, _, split = cut_of(bits, n, R, 0, hq, hkv, hd, [L], 0, 0)
    assert (queries, split) == cut
    tmpl, seen, is_mask = template(R)
    q, k = queries_and_keys((1, R, hq, hd), (1, hkv, L, hd), 61)
    v, kr, vr = rows((1, hkv, L, hd), 64, torch.bfloat16), rows((1, hkv, R, hd), 65, torch.bfloat16), rows((1, hkv, R, hd), 66, torch.bfloat16)
    kr[..., 0] = 0
    out, tol = expected(q, ref.rounded(k, bits)[:, :, FAR:], ref.rounded(v, bits)[:, :, FAR:], kr, vr, [L - FAR], seen, is_mask)
    q, k, v, kr, vr = (t.expand(n, -1, -1, -1).contiguous().cuda() for t in (q, k, v, kr, vr))      # (the sequences are alike)
    cache = make(hkv, hd, n, L, bits)
    bita.kv_write_mx(cache, k, v, i32([0] * n))
    got = bita.tree_attention_mx(tmpl, q, cache, kr, vr, i32([L] * n), L)
    near(got[:1], out, tol)
    assert torch.equal(got, got[:1].expand_as(got))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("peaks", [{}, {70: 23, 130: 25}, {75: 20, 140: 23.5, 210: 25}])
def test_over_prompts(peaks, hd):
    import paper_2401_12522_amd as bita
    T, hq, hkv = 300, 4, 2
    q, k = queries_and_keys((T, hq, hd), (hkv, T, hd), 71, peaks)
    k, v = k.transpose(0, 1).contiguous(), rows((T, hkv, hd), 74, torch.bfloat16)
    out, tol = expected_of_prompts(q[FAR:], k[FAR:], v[FAR:], [0, T - FAR])                         # (the first tokens' own results are left out)
    got = bita.prompt_attention(q.cuda(), k.cuda(), v.cuda(), i32([0, T]))
    near(got[FAR:], out, tol)
