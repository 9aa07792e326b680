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
