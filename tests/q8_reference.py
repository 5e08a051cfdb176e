"""A decoder pass whose layers' matrices and their inputs are 8-bit integers with scales, in float64 numpy: the oracle's pass
with every product of a layer replaced by its 8-bit form.  Test infrastructure; shares no code with the HIP path."""
import numpy as np

import synth
from oracle.model import attend_row, rmsnorm, rope_rotate, silu


def rows_q8(v):
    """Integers and fp32 scales of the rows of v."""
    v = np.asarray(v, np.float64)
    top = np.abs(v).max(1, keepdims=True)
    return np.rint(127 * v / np.where(top > 0, top, 1.0)), (top[:, 0] / 127).astype(np.float32).astype(np.float64)


def linear_q8(v, w):
    (q, s), (qw, sw) = rows_q8(v), rows_q8(w)
    return (q @ qw.T) * s[:, None] * sw


def f32(v):
    return np.asarray(v, np.float32).astype(np.float64)


def forward_rows_q8(model, tokens, is_mask, mask_index, pos, visible_rows, cache_k, cache_v):
    cfg, R = model.cfg, len(tokens)
    Hq, Hkv, hd = cfg.n_heads, cfg.n_kv_heads, cfg.head_dim
    x = np.zeros((R, cfg.d_model))
    for r in range(R):
        if is_mask[r]:
            x[r] = model.w("mask_emb")[mask_index[r]]
        elif tokens[r] >= 0:
            x[r] = model.w("tok_emb")[tokens[r]]
    new_k, new_v = [], []
    for l in range(cfg.n_layers):
        h = rmsnorm(x, model.w("attn_norm", l), cfg.rms_eps)
        q, k, v = (linear_q8(h, model.w(n, l)) for n in ("wq", "wk", "wv"))
        q, k, v = q.reshape(R, Hq, hd), k.reshape(R, Hkv, hd), v.reshape(R, Hkv, hd)
        for r in range(R):
            q[r], k[r] = rope_rotate(q[r], pos[r], cfg.rope_theta), rope_rotate(k[r], pos[r], cfg.rope_theta)
        attn = np.zeros((R, Hq, hd))
        for r in range(R):
            if not is_mask[r] and tokens[r] < 0:
                continue
            ks, vs = [], []
            if is_mask[r] and cfg.n_prompt > 0:
                ks.append(np.transpose(model.w("prompt_k", l), (1, 0, 2)))
                vs.append(np.transpose(model.w("prompt_v", l), (1, 0, 2)))
            ks += [np.asarray(cache_k[l], np.float64), k[list(visible_rows[r])]]
            vs += [np.asarray(cache_v[l], np.float64), v[list(visible_rows[r])]]
            attn[r] = attend_row(q[r], np.concatenate(ks, 0), np.concatenate(vs, 0), Hq, Hkv)
        x = f32(x + linear_q8(synth.bf16_round(attn.reshape(R, Hq * hd)), model.w("wo", l)))
        h = rmsnorm(x, model.w("ffn_norm", l), cfg.rms_eps)
        x = f32(x + linear_q8(silu(linear_q8(h, model.w("w_gate", l))) * linear_q8(h, model.w("w_up", l)), model.w("w_down", l)))
        new_k.append(k)
        new_v.append(v)
    return rmsnorm(x, model.w("final_norm"), cfg.rms_eps) @ model.w("lm_head").T, new_k, new_v
