"""The 8-bit linear layers of a decoder as cases that can be timed and compared.

Four operators, each through the package's public calls:

  norm   h = x + delta (stored), RMSNorm of h times a gain, each row rounded to 8-bit integers with a scale of its own
  gate   silu(gate) * up, rows rounded the same way
  rows   rows of a matrix rounded the same way (an attention output in front of its projection; a weight, one scale a channel)
  gemm   the product of two matrices of 8-bit integers, with the scales of its rows (tokens) and columns (channels)

A row v is held as q = round(127 v / max|v|), ties to even, and the scale s = max|v| / 127: v is about q s.  A row of zeros has
scale 0.  Where such a row is an output, what comes back is q s in 32 bits, beside s.  With `own` false the same is computed in
elementary torch operations.  Values next to a rounding border would come out on either side of it in 32 bits, a whole step
apart, so the plain forms find q in 64 bits; everything else is in 32."""
import math
import random

import torch

own = False


def listed():
    return [
        # One token's output projection at 7B widths: a plain decoding pass, where a call's latency is most of it.
        dict(name="gemm-one-row-7b-o", op="gemm", m=1, n=4096, k=4096, out="f32"),
        # The widest matrix of a 7B layer under a 64-node tree with its mask group.
        dict(name="gemm-68-rows-7b-gate-up", op="gemm", m=68, n=22016, k=4096, out="f32"),
        # The longest sums of the 70B shape, the same tree: one pass over 235 MB of weights.
        dict(name="gemm-68-rows-70b-down", op="gemm", m=68, n=8192, k=28672, out="f32"),
        # Four sequences and some, a vocabulary and a width that no tile divides.
        dict(name="gemm-293-rows-odd-vocabulary", op="gemm", m=293, n=32003, k=5115, out="bf16"),
        # A prompt through the widest matrix of a 70B layer.
        dict(name="gemm-4096-rows-70b-gate-up", op="gemm", m=4096, n=57344, k=8192, out="bf16"),
        # One token between two layers of 7B: launches and latency.
        dict(name="norm-one-row-7b", op="norm", m=1, d=4096, x="f32", delta="f32"),
        # A tree at 70B widths, the residual stream in 32 bits as the verify step keeps it.
        dict(name="norm-68-rows-70b", op="norm", m=68, d=8192, x="f32", delta="f32"),
        # A batch of prompts at 13B widths, residual stream and delta in bf16.
        dict(name="norm-8192-rows-13b", op="norm", m=8192, d=5120, x="bf16", delta="bf16"),
        # Gate and up columns of a tree as the product of the interleaved weight leaves them (tiles of 16).
        dict(name="gate-68-rows-7b", op="gate", m=68, f=11008, x="f32", tile=16),
        # A prompt at 70B widths, all gate columns before all up columns.
        dict(name="gate-4096-rows-70b", op="gate", m=4096, f=28672, x="bf16", tile=0),
        # The attention output of a tree.
        dict(name="rows-68-7b", op="rows", m=68, k=4096, x="bf16"),
        # A weight of a 7B layer, one scale for each channel: done once when a model is loaded.
        dict(name="rows-weight-7b-gate", op="rows", m=11008, k=4096, x="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["gemm", "gemm", "gemm", "norm", "gate", "rows"])
    x = rng.choice(["f32", "bf16"])
    if op == "gemm":
        n, k = _log(rng, 64, 57344), _log(rng, 64, 28672)
        m = _log(rng, 1, max(1, min(4096, 4096 * 57344 * 8192 // (n * k))))
        return dict(op="gemm", m=m, n=n, k=k, out=x)
    if op == "norm":
        d = _log(rng, 64, 16384)
        return dict(op="norm", m=_log(rng, 1, 8192 * 5120 // d), d=d, x=x, delta=rng.choice([x, "f32", "none"]))
    if op == "gate":
        f, tile = _log(rng, 16, 28672), rng.choice([0, 16])
        f = f // 16 * 16 if tile else f
        return dict(op="gate", m=_log(rng, 1, 4096 * 28672 // f), f=f, x=x, tile=tile)
    k = _log(rng, 64, 28672)
    return dict(op="rows", m=_log(rng, 1, 11008 * 4096 // k), k=k, x=x)


_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2, "none": 0}


def _activations(m, k, g, spread=0.5):
    """Rows as a decoder has them: channels of unequal size, a few of them far larger than the rest."""
    x = torch.randn(m, k, device="cuda", generator=g)
    size = torch.exp(spread * torch.randn(k, device="cuda", generator=g))
    size[torch.randint(0, k, (max(1, k // 500),), device="cuda", generator=g)] *= 12
    return x.mul_(size)


def _codes(v):
    """8-bit integers and scales of the rows of v, for inputs that hold them already."""
    s = v.abs().amax(1).clamp_min(1e-30) / 127
    return v.div_(s[:, None]).round_().clamp_(-127, 127).to(torch.int8), s


def _empty_q(m, k):
    """Rows of 8-bit integers, 16 bytes or a multiple apart."""
    return torch.empty((m, (k + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :k]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m, s = case["m"], {"op": case["op"]}
    if case["op"] == "gemm":
        n, k = case["n"], case["k"]
        codes, s["a_scale"] = _codes(_activations(m, k, g))
        s["a"] = _empty_q(m, k).copy_(codes)
        s["w"], s["w_scale"] = _codes(torch.randn(n, k, device="cuda", generator=g).mul_(0.02))
        s["out"] = torch.empty((m, n), dtype=_TYPE[case["out"]], device="cuda")
        if own:                                            # laid out once, when a model is loaded
            import paper_2401_12522_amd as bita
            s["packed"] = bita.pack_weight_q8(s["w"])
        return s
    k = case["d"] if case["op"] == "norm" else case["f"] if case["op"] == "gate" else case["k"]
    s["q"], s["scale"] = _empty_q(m, k), torch.empty(m, dtype=torch.float32, device="cuda")
    if case["op"] == "norm":
        s["x"] = _activations(m, k, g).to(_TYPE[case["x"]])
        s["gain"] = (1 + 0.2 * torch.randn(k, device="cuda", generator=g)).to(torch.bfloat16)
        s["eps"], s["delta"], s["total"] = 1e-5, None, None
        if case["delta"] != "none":
            s["delta"] = _activations(m, k, g).mul_(0.3).to(_TYPE[case["delta"]])
            s["total"] = torch.empty_like(s["x"])
        if m >= 16:                                        # a draft row for which there was no candidate
            s["x"][m // 2] = 0
            if s["delta"] is not None:
                s["delta"][m // 2] = 0
    elif case["op"] == "gate":
        s["x"], s["tile"] = _activations(m, 2 * k, g).to(_TYPE[case["x"]]), case["tile"]
    else:
        s["x"] = _activations(m, k, g).to(_TYPE[case["x"]])
    return s


def _rounded(v):
    """Plain form of the rounding: v in 64 bits -> q s, s."""
    top = v.abs().amax(1, keepdim=True)
    q = torch.round(v * 127 / torch.where(top > 0, top, 1.0))
    return q, top / 127


def _halves(x, tile):
    m, f2 = x.shape
    if tile:
        x = x.view(m, f2 // (2 * tile), 2, tile)
        return x[:, :, 0].reshape(m, f2 // 2), x[:, :, 1].reshape(m, f2 // 2)
    return x[:, : f2 // 2], x[:, f2 // 2:]


def run(s):
    if own:
        import paper_2401_12522_amd as bita
        if s["op"] == "gemm":
            return {"y": bita.gemm_q8(s["a"], s["a_scale"], s["packed"], s["w_scale"], s["w"].shape[0], out=s["out"])}
        if s["op"] == "norm":
            q, scale = bita.norm_q8(s["x"], s["gain"], s["eps"], delta=s["delta"], total=s["total"], q=s["q"], scale=s["scale"])
            return {"y": q * scale[:, None], "scale": scale, "total": s["total"]}
        if s["op"] == "gate":
            q, scale = bita.silu_mul_q8(s["x"], tile=s["tile"], q=s["q"], scale=s["scale"])
        else:
            q, scale = bita.quantize_rows(s["x"], q=s["q"], scale=s["scale"])
        return {"y": q * scale[:, None], "scale": scale}
    if s["op"] == "gemm":
        y = s["a"].float() @ s["w"].float().T
        return {"y": (y * s["a_scale"][:, None] * s["w_scale"]).to(s["out"].dtype)}
    total = None
    if s["op"] == "norm":
        h = s["x"]
        if s["delta"] is not None:
            h = total = (s["x"].float() + s["delta"].float()).to(s["x"].dtype)
        r = torch.rsqrt(h.float().square().mean(1) + s["eps"])
        q, step = _rounded(h.double() * s["gain"].double())     # (a row's factor changes its scale, not its q)
        scale = step[:, 0].float() * r
    else:
        if s["op"] == "gate":
            gate, up = _halves(s["x"], s["tile"])
            gate = gate.double()
            v = gate / (1 + torch.exp(-gate)) * up.double()
        else:
            v = s["x"].double()
        q, step = _rounded(v)
        scale = step[:, 0].float()
    out = {"y": q.float() * scale[:, None], "scale": scale}
    if s["op"] == "norm":
        out["total"] = total
    return out


def work(case):
    m = case["m"]
    if case["op"] == "gemm":
        n, k = case["n"], case["k"]
        return {"bytes": m * k + n * k + 4 * (m + n) + _SIZE[case["out"]] * m * n, "flops": 2 * m * n * k}
    if case["op"] == "norm":
        k, size = case["d"], _SIZE[case["x"]] + _SIZE[case["delta"]] + (_SIZE[case["x"]] if case["delta"] != "none" else 0)
        return {"bytes": m * k * (size + 4) + 2 * k + 4 * m, "flops": 6 * m * k}
    if case["op"] == "gate":
        return {"bytes": m * case["f"] * (2 * _SIZE[case["x"]] + 4) + 4 * m, "flops": 8 * m * case["f"]}
    return {"bytes": m * case["k"] * (_SIZE[case["x"]] + 4) + 4 * m, "flops": 3 * m * case["k"]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "gemm":
        a = s["a"].double().mul_(s["a_scale"].double()[:, None])
        return {"y": torch.matmul(a, s["w"].double().mul_(s["w_scale"].double()[:, None]).T)}
    out = {"total": None}
    if case["op"] == "norm":
        h = s["x"].double()
        if s["delta"] is not None:
            h = out["total"] = h + s["delta"].double()
            h = h.float().to(s["x"].dtype).double()              # what is stored is what is normalised
        v = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["d"] + s["eps"]) * s["gain"].double()
        codes = h * s["gain"].double()                           # the same row but for a positive factor
    elif case["op"] == "gate":
        x, f = s["x"].double(), case["f"]
        j = torch.arange(f, device="cuda")
        at = j // 16 * 32 + j % 16 if case["tile"] else j
        gate = x[:, at]
        codes = v = gate * torch.sigmoid(gate) * x[:, at + (16 if case["tile"] else f)]
    else:
        codes = v = s["x"].double()
    step = v.abs().max(1).values / 127
    top = codes.abs().max(1, keepdim=True).values
    t = codes.abs() * 127 / top.clamp_min(1e-300)
    low = torch.floor(t)
    up = (t - low > 0.5) | ((t - low == 0.5) & (low % 2 == 1))
    out.update(y=(low + up) * torch.sign(codes) * step[:, None], scale=step)
    return out if case["op"] == "norm" else {"y": out["y"], "scale": out["scale"]}
