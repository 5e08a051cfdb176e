"""Causal attention over packed prompts (GPU) against float64 on the CPU; the tolerance is worked out in mx_reference.attention."""
import pytest
import torch

import mx_reference as ref
from test_gpu_kv_mx import i32, rows

pytestmark = pytest.mark.gpu


def starts(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def expected(q, k, v, cu):
    T, hq, hd = q.shape
    hkv = k.shape[1]
    out, tol = torch.zeros(2, T, hq, hd, dtype=torch.float64)
    for a, b in zip(cu, cu[1:]):
        seen = torch.ones(b - a, b - a, dtype=torch.bool).tril()
        for h in range(hq if b > a else 0):
            g = h // (hq // hkv)
            out[a:b, h], tol[a:b, h] = ref.attention(q[a:b, h].double(), k[a:b, g].double(), v[a:b, g].double(), seen)
    return out, tol


def near(got, out, tol):
    off = (got.cpu().double().view(out.shape) - out).abs()
    assert (off <= tol).all(), float((off / tol).max())


def tensors(T, hq, hkv, hd, seed=0):
    return rows((T, hq, hd), seed, torch.bfloat16), rows((T, hkv, hd), seed + 1, torch.bfloat16), rows((T, hkv, hd), seed + 2, torch.bfloat16)


@pytest.mark.parametrize("lens,hq,hkv,hd", [
    ([1], 4, 4, 64), ([2], 4, 2, 128), ([31, 1, 33], 2, 1, 64), ([64], 8, 8, 128), ([65, 0, 63], 12, 4, 64), ([127, 128, 129], 4, 2, 128),
    ([0, 0, 5, 0], 6, 2, 128), ([300], 16, 2, 64), ([511, 17], 5, 1, 128), ([1] * 70 + [0, 40], 1, 1, 64), ([1000], 8, 1, 128), ([257, 640], 40, 40, 64)])
@pytest.mark.parametrize("fused", [False, True])
def test_against_float64(lens, hq, hkv, hd, fused):
    import paper_2401_12522_amd as bita
    cu = starts(lens)
    T = cu[-1] + 3                                                # rows behind the last sequence
    q, k, v = tensors(T, hq, hkv, hd)
    out, tol = expected(q, k, v, cu)
    a = (q.cuda(), k.cuda(), v.cuda())
    if fused:
        x = torch.cat(a, 1)
        a = (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:])
    got = torch.full((T, hq * hd), 5.0, dtype=torch.bfloat16, device="cuda")
    assert bita.prompt_attention(*a, i32(cu), out=got) is got
    near(got[: cu[-1]], out[: cu[-1]], tol[: cu[-1]])
    assert (got[cu[-1]:] == 5).all()


@pytest.mark.parametrize("n", [64, 65, 513, 1100, 3000])
def test_very_many_short_sequences(n):
    """Against the same sequences one call each would give: lengths 0 to 3 and a few of some hundred rows among them."""
    import paper_2401_12522_amd as bita
    lens = [(i * 7) % 4 for i in range(n)]
    for i in (0, n // 2, n - 1):
        lens[i] = 150 + i % 100
    cu = starts(lens)
    q, k, v = tensors(cu[-1], 2, 1, 64)
    out, tol = expected(q, k, v, cu)
    near(bita.prompt_attention(q.cuda(), k.cuda(), v.cuda(), i32(cu)), out, tol)


def test_rows_before_the_first_sequence_and_wide_output_rows():
    import paper_2401_12522_amd as bita
    q, k, v = tensors(60, 4, 2, 64)
    cu = [7, 40, 55]
    out, tol = expected(q, k, v, cu)
    wide = torch.full((60, 4 * 64 + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    bita.prompt_attention(q.cuda(), k.cuda(), v.cuda(), i32(cu), out=wide[:, :256])
    near(wide[7:55, :256], out[7:55], tol[7:55])
    assert (wide[:, 256:] == 5).all() and (wide[:7] == 5).all() and (wide[55:] == 5).all()


def test_ends_outside_the_tokens_are_clamped():
    import paper_2401_12522_amd as bita
    q, k, v = tensors(50, 2, 2, 64)
    for given, meant in (([-9, 20, 2 ** 31 - 1], [0, 20, 50]), ([0, 30, 10, 50], [0, 30, 30, 30]), ([60, 70], [50, 50])):
        got = torch.zeros((50, 128), dtype=torch.bfloat16, device="cuda")
        bita.prompt_attention(q.cuda(), k.cuda(), v.cuda(), i32(given), out=got)
        if meant == [0, 30, 30, 30]:                              # (sequences that go back are not promised anything but to stay inside)
            continue
        out, tol = expected(q, k, v, meant)
        near(got, out, tol)


def test_later_tokens_and_other_sequences_do_not_matter():
    """NaN and infinities in K and V of token j: only its sequence's tokens from j on may notice."""
    import paper_2401_12522_amd as bita
    cu = [0, 70, 200, 230]
    q, k, v = tensors(230, 4, 2, 128)
    q = (q.float() / 8).to(torch.bfloat16)                        # (no probability so small that it is 0: 0 times infinity is NaN)
    out, tol = expected(q, k, v, cu)
    for j in (0, 37, 69, 70, 135, 199, 229):
        k2, v2 = k.clone(), v.clone()
        v2[j, :, 0::3], v2[j, :, 1::3], v2[j, :, 2::3], k2[j] = float("nan"), float("inf"), float("-inf"), float("nan")
        end = next(e for e in cu if e > j)
        for keys in (k, k2):
            got = bita.prompt_attention(q.cuda(), keys.cuda(), v2.cuda(), i32(cu)).cpu().double().view(out.shape)
            near(torch.cat([got[:j], got[end:]]), torch.cat([out[:j], out[end:]]), torch.cat([tol[:j], tol[end:]]))
            hit = got[j:end]
            if keys is k2:
                assert hit.isnan().all()
            else:
                assert hit[..., 0::3].isnan().all() and (hit[..., 1::3] == float("inf")).all() and (hit[..., 2::3] == float("-inf")).all()


def test_large_scores_and_a_moving_maximum():
    import paper_2401_12522_amd as bita
    q, k, v = tensors(500, 2, 1, 128)
    k = (k.float() * torch.linspace(0.1, 12, 500)[:, None, None]).to(torch.bfloat16)
    out, tol = expected(q, k, v, [0, 500])
    near(bita.prompt_attention(q.cuda(), k.cuda(), v.cuda(), i32([0, 500])), out, tol)


def test_long_prompt_rows_far_apart():
    """Offsets beyond 2^31 elements: rows of a product so wide that the last ones lie there."""
    import paper_2401_12522_amd as bita
    T, ld = 700, 4_000_000
    big = torch.zeros((T, ld), dtype=torch.bfloat16, device="cuda")
    q, k, v = tensors(T, 2, 1, 64)
    x = big[:, -256:].unflatten(1, (4, 64))
    x[:, :2], x[:, 2:3], x[:, 3:] = q.cuda(), k.cuda(), v.cuda()
    out, tol = expected(q, k, v, [0, 690])
    got = bita.prompt_attention(x[:, :2], x[:, 2:3], x[:, 3:], i32([0, 690]))
    near(got[:690], out[:690], tol[:690])


def test_replayed_from_a_graph():
    import paper_2401_12522_amd as bita
    cu = i32([0, 150, 400])
    q, k, v = (t.cuda() for t in tensors(400, 4, 2, 128))
    out = torch.zeros((400, 512), dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        bita.prompt_attention(q, k, v, cu, out=out)
    for turn in range(3):
        q.copy_(rows(q.shape, 60 + turn, torch.bfloat16))
        cu.copy_(i32([0, 100 + 50 * turn, 399]))
        out.zero_()
        g.replay()
        want = torch.zeros_like(out)
        bita.prompt_attention(q, k, v, cu, out=want)
        assert torch.equal(out, want)
