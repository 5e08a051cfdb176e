"""Attention over the small cache and over prompts (GPU) where values are large and the largest scores come late: the weights are relative to a
reference, and their sums with values up to the size that the calls promise have to stay finite wherever it lies."""
import math

import pytest
import torch

import mx_reference as ref
from test_gpu_kv_mx import i32, make, rows
from test_gpu_prompt_attention import expected as expected_of_prompts, starts
from test_gpu_tree_attention_mx import BITS, cut_of, expected, near, template

pytestmark = pytest.mark.gpu
LARGEST = 2.0 ** 99                                               # 2^108 / (keys that a query sees), of which there are up to 398 here


def queries_and_keys(q_shape, k_shape, peaks, seed):
    """Scores near 0, but for keys `peaks` {slot: octaves}: axis -2 of the keys is their slot."""
    hd = q_shape[-1]
    side = torch.where(rows((hd,), seed) > 0, 1.0, -1.0)
    q = side + 0.3 * rows(q_shape, seed + 1).clamp(-1, 1)
    k = 0.1 * rows(k_shape, seed + 2).clamp(-1, 1)
    for slot, octaves in peaks.items():
        k[..., slot, :] = side * octaves * math.log(2) / math.sqrt(hd)
    return q.to(torch.bfloat16), k.to(torch.bfloat16)


def values(shape, seed):
    x = rows(shape, seed)
    return (torch.sign(x) * (0.5 + 0.5 * torch.tanh(x.abs())) * LARGEST).to(torch.bfloat16)


@BITS
@pytest.mark.parametrize("n,R,hq,hkv,hd,cut", [
    (1, 1, 8, 2, 128, (16, False)), (1, 3, 4, 2, 64, (16, False)), (8, 20, 32, 16, 64, (32, False)), (17, 68, 64, 2, 64, (128, False)), (9, 68, 64, 4, 128, (128, False))])
@pytest.mark.parametrize("peaks", [{70: 20, 130: 58}, {64: 59}, {40: 30, 150: 57, 200: 59, 310: 110}])
def test_over_the_cache(bits, n, R, hq, hkv, hd, cut, peaks):
    import paper_2401_12522_amd as bita
    L = 330
    queries, _, split = cut_of(bits, n, R, 0, hq, hkv, hd, [L], 0, 0)
    assert (queries, split) == cut
    tmpl, seen, is_mask = template(R)
    q, k = queries_and_keys((1, R, hq, hd), (1, hkv, L, hd), peaks, 31)
    v, kr, vr = values((1, hkv, L, hd), 34), rows((1, hkv, R, hd), 35, torch.bfloat16), values((1, hkv, R, hd), 36)
    out, tol = expected(q, ref.rounded(k, bits), ref.rounded(v, bits), kr, vr, [L], seen, is_mask)
    q, k, v, kr, vr = (t.expand(n, -1, -1, -1).contiguous().cuda() for t in (q, k, v, kr, vr))      # (the sequences are alike)
    cache = make(hkv, hd, n, L, bits)
    bita.kv_write_mx(cache, k, v, i32([0] * n))
    got = bita.tree_attention_mx(tmpl, q, cache, kr, vr, i32([L] * n), L)
    near(got[:1], out, tol)
    assert torch.equal(got, got[:1].expand_as(got))


@BITS
def test_over_the_cache_in_shares(bits):
    """Peaks in several shares, in tiles that are not their shares' first."""
    import paper_2401_12522_amd as bita
    R, hq, hkv, hd, L = 130, 16, 1, 128, 6000
    assert cut_of(bits, 1, R, 0, hq, hkv, hd, [L], 0, 0) == (128, 4, True)
    tmpl, seen, is_mask = template(R)
    q, k = queries_and_keys((1, R, hq, hd), (1, hkv, L, hd), {500: 40, 3100: 50, 5990: 59}, 41)
    v, kr, vr = values((1, hkv, L, hd), 44), rows((1, hkv, R, hd), 45, torch.bfloat16), values((1, hkv, R, hd), 46)
    v, vr = v * 2.0 ** -4, vr * 2.0 ** -4                         # (6130 keys)
    out, tol = expected(q, ref.rounded(k, bits), ref.rounded(v, bits), kr, vr, [L], seen, is_mask)
    cache = make(hkv, hd, 1, L, bits)
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), i32([0]))
    near(bita.tree_attention_mx(tmpl, q.cuda(), cache, kr.cuda(), vr.cuda(), i32([L]), L), out, tol)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens,peaks", [([400], {70: 20, 130: 58}), ([400], {64: 59}), ([400], {40: 30, 150: 57, 200: 59, 310: 110, 390: 118}), ([90, 200], {70: 40, 160: 59, 250: 90})])
def test_over_prompts(lens, peaks, hd):
    import paper_2401_12522_amd as bita
    cu, hq, hkv = starts(lens), 4, 2
    T = cu[-1]
    q, k = queries_and_keys((T, hq, hd), (hkv, T, hd), peaks, 51)
    k, v = k.transpose(0, 1).contiguous(), values((T, hkv, hd), 54)
    out, tol = expected_of_prompts(q, k, v, cu)
    near(bita.prompt_attention(q.cuda(), k.cuda(), v.cuda(), i32(cu)), out, tol)
