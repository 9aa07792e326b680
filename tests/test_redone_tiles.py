"""Prompt calls whose tiles are done once more, for values that are not finite and that some of a tile's rows do not see: bad items are
reported once all the same."""
from __future__ import annotations

import math

import numpy as np
import pytest

from test_attn_ops import Cache, _i32


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("n", [2, 32, 33])
def test_bad_items_are_counted_once(dtype, window, n):
    """Up to 32 entries (planned by the tiles themselves) and more (by a list), with enough rows that no tile is split; the last entry names an empty
    slot, the one before has more rows than its chain holds tokens."""
    import torch
    from paper_2605_22416_b200 import binding as B
    hk, hq, dim, bad = 8, 32, 64, 1 if n == 2 else 2
    good = n - bad
    new = [max(40, 1600 // good)] * good
    c = Cache([a + 5 for a in new], hk, dim, 16, dtype, seed=n)
    kv = c.rows[0].clone()
    kv[1, -1] = math.nan                                  # seen by the last row alone
    c.ctx.scatter_kv(c.layer, _i32([0]), None, 1, kv[0].contiguous(), kv[1].contiguous())
    reqs, lens = list(range(good)) + [0, good][-bad:], new + [new[0] + 6, 3][-bad:]
    cu, tot = np.concatenate([[0], np.cumsum(lens)]), sum(lens)
    q, _ = c.queries(tot, hq)
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=0.125)
    ws, size = c.workspace(desc, n)
    out = torch.full((tot, hq, dim), 7.0, dtype=c.dt, device="cuda")
    args = (_i32(reqs), n, _i32(cu), tot, q, out, None, ws, size)
    if window:
        c.ctx.attn_window_prompt(c.layer, desc, window, 0, *args)
    else:
        c.ctx.attn_prompt(c.layer, desc, *args)
    assert torch.isnan(out[new[0] - 1]).all() and torch.isfinite(out[: new[0] - 1]).all() and torch.isfinite(out[new[0]:]).all()
    assert (out[cu[good]:] == 7).all() and c.ctx.stats()["error_count"] == bad
    c.ctx.close()
