"""Scores that are no number in attention over the small cache, in every cut of a launch (GPU): what sees one is NaN, whatever shares the keys are split into,
and nothing else changes."""
import pytest
import torch

from test_gpu_kv_mx import i32
from test_gpu_tree_attention_mx import BITS, CUTS, case, near

pytestmark = pytest.mark.gpu
EVERY_CUT = pytest.mark.parametrize("n,R,masks,hq,hkv,hd,ctx,page,P", CUTS)
NAN = float("nan")


def nan_there(got, out, tol, where):
    """NaN in all columns of the queries `where` [n][R][hq], as expected elsewhere."""
    got = got.cpu().double().view(out.shape)
    assert where.any() and torch.isnan(got[where]).all()
    got[where] = out[where]
    near(got, out, tol)


@BITS
@EVERY_CUT
def test_a_query_that_is_no_number(bits, n, R, masks, hq, hkv, hd, ctx, page, P):
    """Every score of the query is NaN, in every share."""
    call, (out, tol), (cache, q, *_) = case(n, R, masks, hq, hkv, hd, bits, ctx, page, P, seed=17)
    where = torch.zeros(n, R, hq, dtype=torch.bool)
    where[n // 2, R // 2, hq - 1] = where[0, R - 1, 0] = True
    q[where] = NAN
    nan_there(call(), out, tol, where)


@BITS
@EVERY_CUT
def test_a_row_whose_key_is_no_number(bits, n, R, masks, hq, hkv, hd, ctx, page, P):
    """The last token row's own key, which may be all that a share holds for a query."""
    call, (out, tol), (cache, q, kr, vr, _, _, tmpl, seen, _) = case(n, R, masks, hq, hkv, hd, bits, ctx, page, P, seed=18)
    at = R - masks - 1
    kr[n - 1, :, at] = NAN
    where = torch.zeros(n, R, hq, dtype=torch.bool)
    where[n - 1, seen[:, at]] = True
    nan_there(call(), out, tol, where)


@BITS
@EVERY_CUT
def test_cached_keys_that_are_no_numbers(bits, n, R, masks, hq, hkv, hd, ctx, page, P):
    """All cached keys of one sequence and K/V head: whole shares of nothing else."""
    import paper_2401_12522_amd as bita
    call, (out, tol), (cache, q, kr, vr, ck, cv, *_) = case(n, R, masks, hq, hkv, hd, bits, ctx, page, P, seed=19)
    b = max(range(n), key=lambda i: ctx[i])
    k, v = ck.to(torch.bfloat16), cv.to(torch.bfloat16)         # (what is there already, exact in bf16)
    k[b, 0] = NAN
    bita.kv_write_mx(cache, k.cuda(), v.cuda(), i32([0] * n), i32([ctx[b] if i == b else 0 for i in range(n)]))
    where = torch.zeros(n, R, hq, dtype=torch.bool)
    where[b, :, : hq // hkv] = True
    nan_there(call(), out, tol, where)
