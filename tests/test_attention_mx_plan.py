"""How attention over the small cache is cut into workgroups, on the host alone."""
import os

import pytest


def longest_share(batch, rows, heads, kv_heads, bits, hint, n_prompt=0):
    """Where all sequences are as long as the hint: the turns of the longest share over those of an even division, from the plan and the rule by which the kernels cut
    lengths into shares (one size for all of them, the smallest at which they are enough)."""
    from paper_2401_12522_amd import binding, build
    if not os.path.exists(build.LIB_PATH):
        build.build_library()
    plan = binding.tree_attention_mx_plan_info(batch, rows, heads, kv_heads, 128, bits, hint, n_prompt)
    keys, turn = (64, 1) if plan["queries"] == 128 else (32, plan["waves"])
    tiles = -(-rows * (heads // kv_heads) // plan["queries"])
    shares = plan["workgroups"] // (kv_heads * tiles)
    assert plan["workgroups"] == shares * kv_heads * tiles and plan["splits"] == -(-shares // batch)
    turns = -(-sum(-(-n // keys) for n in (hint, n_prompt, rows)) // turn)
    if shares == batch:
        return 1.0
    size = next(p for p in range(1, turns + 1) if batch * -(-turns // p) <= shares)
    return size * shares / (turns * batch)


@pytest.mark.parametrize("batch,rows,heads,kv_heads,bits,hint,n_prompt", [
    (17, 1, 64, 8, 4, 8192, 0), (18, 1, 64, 8, 4, 8192, 0), (20, 1, 64, 8, 4, 8192, 0), (17, 1, 64, 8, 8, 8192, 0), (20, 1, 64, 8, 8, 8192, 0), (33, 1, 64, 8, 8, 8192, 0),
    (40, 1, 64, 8, 8, 8192, 0), (5, 1, 32, 32, 4, 4096, 0), (5, 1, 32, 32, 8, 4096, 0), (9, 1, 32, 32, 8, 4096, 0), (4, 68, 64, 8, 4, 3000, 16), (4, 68, 64, 8, 8, 3000, 16)])
def test_shares_of_equal_lengths(batch, rows, heads, kv_heads, bits, hint, n_prompt):
    """Batches for which one share more or less a sequence matters most: with few more shares than sequences, alike ones still have one each."""
    assert longest_share(batch, rows, heads, kv_heads, bits, hint, n_prompt) < 1.49
