"""Attention over the paged KV chains where some of the chain must not count: values that a row does not see, scores of
minus infinity, and weights far below the largest one.

Tolerance, entry by entry.  out_i = sum_j w_j v_j; a weight is rounded to the 16 bits of V (eps/2 relative) and the output once
(eps/2); the exponentials (2^-18.6, or 2^-22) and the 32-bit sums stay inside another eps/2 of either type.  So an entry is off by at
most 3 * eps/2 * sum_j w_j |v_j|, whatever the signs.  The log-sum: 2^-18 absolute plus 2^-20 relative."""
from __future__ import annotations

import math

import numpy as np
import pytest

from test_attn_ops import NONE, Cache, _i32


def _exact(q, kv, scale, past):
    """q [n, q_heads, dim] at positions past + i over kv [2, L, kv_heads, dim] -> out, lse, sum_j w_j |v_j| in 64 bits; a
    weight of zero (a token that is not seen) counts as nothing, whatever its value."""
    import torch
    rep = q.shape[1] // kv.shape[2]
    K, V = (x.double().repeat_interleave(rep, 1) for x in kv)
    j, i = torch.arange(kv.shape[1], device="cuda"), torch.arange(q.shape[0], device="cuda") + past
    z = torch.einsum("ihd,jhd->hij", q.double(), K) * scale
    z.masked_fill_(j[None] > i[:, None], -math.inf)
    lse = torch.logsumexp(z, -1)
    w = (z - lse[..., None]).exp()
    return torch.einsum("hij,jhd->ihd", w, V), lse.transpose(0, 1), torch.einsum("hij,jhd->ihd", w, V.abs())


def _close(out, lse, want, want_lse, size, what, keep=None):
    import torch
    d = (out.double() - want).abs() - 3 * torch.finfo(out.dtype).eps / 2 * size
    if keep is not None:
        d = d[keep]
    assert d.numel() == 0 or float(d.max()) <= 0, f"{what}: {float(d.max()):.3g} too far off"        # (a NaN fails too)
    assert float(((lse.double() - want_lse).abs() - 2.0 ** -20 * want_lse.abs()).max()) <= 2.0 ** -18, f"{what}: log-sum"


SHAPES = [
    # held, new, kv_heads, group, dim, page
    ([300, 50], [300, 50], 2, 2, 64, 16),
    ([700], [300], 1, 1, 128, 16),                    # tokens split over the SMs
    ([300, 33], [300, 33], 8, 16, 64, 32),            # more tiles than SMs
    ([260, 129], [129, 129], 2, 3, 128, 24),          # groups that do not divide a tile
    ([90] * 40, [40] * 40, 2, 8, 128, 16),            # a list with a plan of its own
    ([400] * 20, [350] * 20, 8, 4, 128, 128),         # several tiles an SM
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, "lowest"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_a_value_counts_for_the_rows_that_see_it_and_no_others(case, value, dtype):
    import torch
    from paper_2605_22416_b200 import binding as B
    held, new, hk, group, dim, page = SHAPES[case]
    c = Cache(held, hk, dim, page, dtype, seed=40 + case)
    lowest = torch.finfo(c.dt).min
    hq, scale, tot = hk * group, dim ** -0.5, sum(new)
    cu = np.concatenate([[0], np.cumsum(new)])
    planted = [(0, held[0] - x, i % hk, 5 * i + 1) for i, x in enumerate([1, 2, 17, 40, min(129, held[0] - 3), held[0]])]
    planted += [(0, held[0] // 16 * 16 - x, x % hk, 30 + x) for x in (9, 10, 25)]           # tokens 7, 6 and 7 of 16
    planted += [(len(held) - 1, held[-1] // 2, hk - 1, dim - 1)]
    clean = {r: kv.clone() for r, kv in c.rows.items()}
    for r, p, h, x in planted:
        c.rows[r][1, p, h, x] = lowest if value == "lowest" else value
        clean[r][1, p, h, x] = lowest if value == "lowest" else 0
    for r in {p[0] for p in planted}:
        c.ctx.scatter_kv(c.layer, _i32([r]), None, 1, c.rows[r][0].contiguous(), c.rows[r][1].contiguous())
    q, _ = c.queries(tot, hq)
    out, lse = torch.zeros(tot, hq, dim, dtype=c.dt, device="cuda"), torch.zeros(tot, hq, device="cuda")
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale)
    ws, size = c.workspace(desc, len(held))
    c.ctx.attn_prompt(c.layer, desc, _i32(range(len(held))), len(held), _i32(cu), tot, q, out, lse, ws, size)
    for r in range(len(held)):
        a, b = cu[r], cu[r + 1]
        past = held[r] - new[r]
        want, want_lse, mass = _exact(q[a:b], clean[r], scale, past)
        keep = torch.ones(b - a, hq, dim, dtype=torch.bool, device="cuda")
        if value != "lowest":
            for s, p, h, x in planted:
                if s == r:
                    rows = slice(max(0, p - past), b - a)
                    heads = slice(h * group, (h + 1) * group)
                    keep[rows, heads, x] = False
                    got = out[a:b][rows, heads, x]
                    assert (got.isnan() if math.isnan(value) else got == value).all(), f"slot {r}, token {p}: not seen"
        _close(out[a:b], lse[a:b], want, want_lse, mass, f"slot {r}", keep)
    assert c.ctx.stats()["error_count"] == 0
    c.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("call", ["prompt", "decode", "prefix"])
def test_scores_of_minus_infinity(call, dtype):
    """Tokens whose score is -inf weigh nothing, wherever they stand; a row that sees no others has no average: NaN, and -inf
    for its log-sum."""
    import torch
    from paper_2605_22416_b200 import binding as B
    held, dim, hq, scale = [300, 40, 100, 150], 64, 4, 0.125
    c = Cache(held, 2, dim, 16, dtype, seed=60)
    off = {0: (0, 140), 1: (0, 40), 2: (20, 90), 3: (0, 135)}            # slot 1: all of it
    for r, (a, b) in off.items():
        c.rows[r][0, a:b, :, 0] = -math.inf
        c.ctx.scatter_kv(c.layer, _i32([r]), None, 1, c.rows[r][0].contiguous(), c.rows[r][1].contiguous())
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale)
    ws, size = c.workspace(desc, 4)
    if call == "prompt":
        n, cu = 3, [0, 300, 340, 440]
        parts = [(cu[r], cu[r + 1], c.rows[r], 0) for r in range(3)]
    else:
        n = 3
        parts = [(r, r + 1, torch.cat([c.rows[3], c.rows[r]], 1) if call == "prefix" else c.rows[r], None) for r in range(3)]
    tot = parts[-1][1]
    q, _ = c.queries(tot, hq)
    q[:, :, 0] = 1
    out, lse = torch.zeros(tot, hq, dim, dtype=c.dt, device="cuda"), torch.zeros(tot, hq, device="cuda")
    if call == "prompt":
        c.ctx.attn_prompt(c.layer, desc, _i32(range(3)), 3, _i32(cu), tot, q, out, lse, ws, size)
    else:
        c.ctx.attn_decode(c.layer, desc, _i32(range(3)), 3, 3 if call == "prefix" else NONE, q, out, lse, ws, size)
    for r, (a, b, kv, past) in enumerate(parts):
        want, want_lse, mass = _exact(q[a:b], kv, scale, kv.shape[1] - 1 if past is None else past)
        none = want_lse == -math.inf
        assert (out[a:b][none].isnan()).all() and (lse[a:b][none] == -math.inf).all(), f"slot {r}: rows that see nothing"
        if (~none).any():
            _close(out[a:b][~none], lse[a:b][~none], want[~none], want_lse[~none], mass[~none], f"slot {r}")
    if call != "prefix":
        assert lse[parts[1][0]:parts[1][1]].isinf().all()
    c.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("call", ["prompt", "decode", "prefix"])
def test_many_small_weights_beside_a_large_one(call, dtype):
    """A first token that takes nearly all the weight and has no value, and 20 000 behind it at 2^-25.5 of its weight each: the
    output is all theirs."""
    import torch
    from paper_2605_22416_b200 import binding as B
    L, dim, hq = 20001, 64, 4
    c = Cache([L, 1] + [0] * 300, 1, dim, 64, dtype, seed=61)
    kv = torch.zeros_like(c.rows[0])
    kv[0, 0, :, 0] = 4.0
    kv[1, 1:] = 1.0 + 0.25 * torch.rand(L - 1, 1, dim, device="cuda", generator=c.gen).to(c.dt)
    c.rows[0] = kv
    c.rows[1] = torch.zeros_like(c.rows[1])
    for r in (0, 1):
        c.ctx.scatter_kv(c.layer, _i32([r]), None, 1, c.rows[r][0].contiguous(), c.rows[r][1].contiguous())
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=25.5 * math.log(2) / 4)
    # single tokens: a batch so large that an entry stays on a few SMs (a part without the first token has weights of its own)
    rows = 3 if call == "prompt" else 300
    n = 1 if call == "prompt" else rows
    ws = torch.empty(c.ctx.attn_workspace_bytes(desc, n), dtype=torch.uint8, device="cuda")
    size = ws.numel()
    q = torch.zeros(rows, hq, dim, dtype=c.dt, device="cuda")
    q[:, :, 0] = 1.0
    out, lse = torch.zeros(rows, hq, dim, dtype=c.dt, device="cuda"), torch.zeros(rows, hq, device="cuda")
    if call == "prompt":
        c.ctx.attn_prompt(c.layer, desc, _i32([0]), 1, _i32([0, 3]), 3, q, out, lse, ws, size)
    else:
        c.ctx.attn_decode(c.layer, desc, _i32([1 if call == "prefix" else 0] * n), n, 0 if call == "prefix" else NONE, q, out, lse, ws, size)
    kv = torch.cat([c.rows[0], c.rows[1]], 1) if call == "prefix" else c.rows[0]
    rows = min(rows, 3)
    want, want_lse, mass = _exact(q[:rows], kv, desc.scale, kv.shape[1] - (rows if call == "prompt" else 1))
    assert 3e-4 < float(want.min()) and float(want.max()) < 1e-3
    if n > 1:
        assert torch.equal(out[:1].expand_as(out).isfinite(), out.isfinite()) and float((out.double() - want[:1]).abs().max()) < 1e-5
    _close(out[:rows], lse[:rows], want, want_lse, mass, call)
    c.ctx.close()


@pytest.mark.gpu
def test_values_near_the_largest():
    """A score 7.5 (in log2 units) above those of the tokens before it, with a value of 2^126, in tiles that the running maximum stays
    behind in: what the output is."""
    import torch
    from paper_2605_22416_b200 import binding as B
    L, dim, hk, hq = 300, 64, 8, 128              # more tiles than SMs: tokens are not split
    c = Cache([L], hk, dim, 16, "bfloat16", seed=62)
    kv = torch.zeros_like(c.rows[0])
    kv[0, 200, :, 0] = 4.0
    kv[1] = 1.0
    kv[1, 200] = 2.0 ** 126
    c.ctx.scatter_kv(c.layer, _i32([0]), None, 1, kv[0].contiguous(), kv[1].contiguous())
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=7.5 * math.log(2) / 4)
    ws, size = c.workspace(desc, 1)
    q = torch.zeros(L, hq, dim, dtype=c.dt, device="cuda")
    q[:, :, 0] = 1.0
    out, lse = torch.zeros(L, hq, dim, dtype=c.dt, device="cuda"), torch.zeros(L, hq, device="cuda")
    c.ctx.attn_prompt(c.layer, desc, _i32([0]), 1, _i32([0, L]), L, q, out, lse, ws, size)
    want, want_lse, mass = _exact(q, kv, desc.scale, 0)
    _close(out, lse, want, want_lse, mass, "prompt")
    c.ctx.close()
