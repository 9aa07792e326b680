"""Attention over the paged KV chains (avmp_attn_prompt, avmp_attn_decode) against the formula in 64 bits.

Tolerances.  Scores are 32-bit sums of exact products; exponentials are good to a few 2^-22.  A weight w_j is rounded to the 16
bits of V (at most eps/2 relative), so an output moves by sum_j d_j w_j v_j with |d_j| <= eps/2; V has independent entries of
random sign here, so do the d_j w_j v_j, and both that sum and the output sum_j w_j v_j have the size of sqrt(sum_j w_j^2): eps/2
of the output's norm.  The denominator is summed from the weights before rounding; their mean rounding is again at most eps/2.
With the output's own rounding: 3 * eps/2 norm-wise.  Single rows have 64 entries or more, for which a factor of 4 is ample.
The log-sum is not rounded to 16 bits: 2^-18 absolute plus 2^-20 relative.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import pytest

from paper_2605_22416_b200 import workloads as W

NONE = 0xFFFFFFFF


def _i32(x):
    import torch
    return torch.tensor(np.asarray(x, np.int64).astype(np.uint32).view(np.int32), device="cuda")


class Cache:
    """A context with the given chains, filled through the scatter; freed pages in between, so chains are out of order.
    `rows[r]`: K and V of a slot, [2, held, kv_heads, dim]."""

    def __init__(self, held, kv_heads, dim, page, dtype, layer=1, seed=0, scale=1.0):
        import torch
        from paper_2605_22416_b200 import binding as B
        self.dt, self.layer, self.held = getattr(torch, dtype), layer, held
        m = SimpleNamespace(n_attn_layers=3, n_ssm_layers=1, page_tokens=page, kv_heads=kv_heads, head_dim=dim, kv_elem_bytes=2,
                            ssm_state_elems=64, ssm_conv_elems=4, ssm_elem_bytes=4)
        slots = len(held) + 3
        max_pages = max(-(-h // page) for h in held) + 1
        u_kv = 3 * 2 * page * kv_heads * dim * 2
        pages = sum(-(-h // page) for h in held) + 8
        arena = torch.empty(pages * u_kv + (slots + 2) * 1088, dtype=torch.uint8, device="cuda")
        arena.view(torch.int16).fill_(-1)          # 0xFFFF is a NaN of both types: what nobody wrote must not matter
        self.ctx = B.Context(m, arena.numel(), (slots + 1) * 288 / arena.numel(), 4, max_requests=slots, max_pages=max_pages,
                             migration_enabled=False, arena=arena)
        st = np.zeros(slots, np.uint32)
        rng = np.random.default_rng(seed)
        if len(held) > 1:                          # scramble the free list first
            few = [min(h, 2 * page) for h in held]
            self.ctx.step_host(W.make_ops(W.OP_ADMIT, np.arange(len(held)), few), len(held), st)
            self.ctx.step_host(W.make_ops(W.OP_FINISH, rng.permutation(len(held)), 0), len(held), st)
        order = rng.permutation([i for i, h in enumerate(held) if h])
        self.ctx.step_host(W.make_ops(W.OP_ADMIT, order, np.asarray(held)[order]), len(order), st)
        assert (st[:len(order)] == 0).all(), st
        gen = torch.Generator("cuda").manual_seed(seed)
        self.rows = {}
        for r, h in enumerate(held):
            if h:
                kv = (torch.randn(2, h, kv_heads, dim, device="cuda", generator=gen) * scale).to(self.dt)
                self.ctx.scatter_kv(layer, _i32([r]), None, 1, kv[0].contiguous(), kv[1].contiguous())
                self.rows[r] = kv
        self.gen = gen
        self.dim, self.kv_heads = dim, kv_heads

    def queries(self, n, q_heads, scale=1.5, pad=0):
        import torch
        width = q_heads * self.dim
        buf = (torch.randn(n, width + pad, device="cuda", generator=self.gen) * scale).to(self.dt)
        return buf[:, :width].unflatten(1, (q_heads, self.dim)), (width + pad) * 2

    def workspace(self, desc, n):
        import torch
        size = self.ctx.attn_workspace_bytes(desc, n)
        assert size > 0
        return torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda"), size


def _exact(q, kv, scale, past):
    """q [n, q_heads, dim] at positions past + i over kv [2, L, kv_heads, dim] -> out, lse in 64 bits."""
    import torch
    rep = q.shape[1] // kv.shape[2]
    K, V = (x.double().repeat_interleave(rep, 1) for x in kv)
    z = torch.einsum("ihd,jhd->hij", q.double(), K) * scale
    j, i = torch.arange(kv.shape[1], device="cuda"), torch.arange(q.shape[0], device="cuda") + past
    z.masked_fill_(j[None] > i[:, None], -math.inf)
    lse = torch.logsumexp(z, -1)
    return torch.einsum("hij,jhd->ihd", (z - lse[..., None]).exp(), V), lse.transpose(0, 1)


def _check(out, lse, want, want_lse, what):
    import torch
    assert torch.isfinite(out).all() and torch.isfinite(lse).all(), what
    tol = 3 * torch.finfo(out.dtype).eps / 2
    err = float((out.double() - want).norm() / want.norm())
    assert err <= tol, f"{what}: relative error {err:.3g} over {tol:.3g}"
    row = (out.double() - want).norm(dim=-1) / want.norm(dim=-1)
    assert float(row.max()) <= 4 * tol, f"{what}: a row is {float(row.max()):.3g} off"
    d = (lse.double() - want_lse).abs() - 2.0 ** -20 * want_lse.abs()
    assert float(d.max()) <= 2.0 ** -18, f"{what}: log-sum off by {float(d.max()):.3g}"


DECODE = [
    # held, kv_heads, group, dim, page
    ([1], 1, 1, 64, 16),
    ([16, 17, 15, 1, 200], 8, 4, 128, 16),
    ([33, 1000, 5], 8, 1, 128, 16),
    ([129, 64, 3000], 4, 8, 64, 32),
    ([77, 2], 2, 16, 128, 64),
    ([500, 31, 8, 9], 1, 40, 128, 16),
    ([250, 7], 5, 3, 64, 24),
    ([100, 300], 3, 64, 64, 16),
    ([90, 1, 40], 16, 2, 128, 8),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(DECODE)))
def test_decode(dtype, case):
    import torch
    from paper_2605_22416_b200 import binding as B
    held, hk, group, dim, page = DECODE[case]
    c = Cache(held, hk, dim, page, dtype, seed=case)
    hq = hk * group
    reqs = list(reversed(range(len(held)))) + [0]                # slots may repeat
    n = len(reqs)
    q, qs = c.queries(n, hq, pad=8)
    scale = dim ** -0.5
    out = torch.full((n + 1, hq * dim + 16), 7.0, dtype=c.dt, device="cuda")
    lse = torch.full((n + 1, hq), 7.0, device="cuda")
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale, q_stride_bytes=qs, out_stride_bytes=(hq * dim + 16) * 2)
    ws, size = c.workspace(desc, n)
    for _ in range(2):
        c.ctx.attn_decode(c.layer, desc, _i32(reqs), n, NONE, q, out, lse, ws, size)
    got = out[:, :hq * dim].reshape(n + 1, hq, dim)
    for i, r in enumerate(reqs):
        want, want_lse = _exact(q[i:i + 1], c.rows[r], scale, held[r] - 1)
        _check(got[i:i + 1], lse[i:i + 1], want, want_lse, f"entry {i} (slot {r}, {held[r]} tokens)")
    assert (out[n:] == 7).all() and (lse[n:] == 7).all() and (out[:, hq * dim:] == 7).all()
    assert c.ctx.stats()["error_count"] == 0
    c.ctx.close()


PREFIX = [
    # prefix, held, kv_heads, group, dim, page
    (1, [1], 1, 1, 64, 16),
    (127, [3, 40, 16], 8, 4, 128, 16),
    (2000, [100, 1, 17, 300, 64] * 9, 2, 8, 128, 16),
    (300, [5] * 70, 4, 4, 64, 32),
    (129, [33, 2], 1, 40, 128, 8),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(PREFIX)))
def test_decode_behind_a_shared_prefix(dtype, case):
    import torch
    from paper_2605_22416_b200 import binding as B
    prefix, held, hk, group, dim, page = PREFIX[case]
    n = len(held)
    c = Cache(held + [prefix], hk, dim, page, dtype, seed=10 + case)
    hq = hk * group
    q, _ = c.queries(n, hq)
    scale = -(dim ** -0.5) if case == 1 else dim ** -0.5
    out, lse = torch.zeros(n, hq, dim, dtype=c.dt, device="cuda"), torch.zeros(n, hq, device="cuda")
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale)
    ws, size = c.workspace(desc, n)
    c.ctx.attn_decode(c.layer, desc, _i32(range(n)), n, n, q, out, lse, ws, size)
    for r in range(n):
        want, want_lse = _exact(q[r:r + 1], torch.cat([c.rows[n], c.rows[r]], 1), scale, prefix + held[r] - 1)
        _check(out[r:r + 1], lse[r:r + 1], want, want_lse, f"slot {r}")
    assert c.ctx.stats()["error_count"] == 0
    c.ctx.close()


PROMPT = [
    # held, new, kv_heads, group, dim, page
    ([1], [1], 1, 1, 64, 16),
    ([5, 130, 64, 33], [5, 130, 64, 33], 8, 4, 128, 16),
    ([300, 40, 1000], [300, 0, 17], 2, 8, 128, 16),
    ([700], [700], 4, 1, 64, 32),
    ([513, 200], [256, 199], 1, 40, 128, 8),
    ([129, 128, 127], [129, 128, 127], 2, 3, 128, 64),
    ([2500], [3], 2, 2, 128, 16),
    ([3000, 70], [12, 1], 1, 16, 64, 24),
    ([400] * 20, [150] * 20, 8, 4, 128, 128),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(PROMPT)))
def test_prompt(dtype, case):
    import torch
    from paper_2605_22416_b200 import binding as B
    held, new, hk, group, dim, page = PROMPT[case]
    c = Cache(held, hk, dim, page, dtype, seed=20 + case)
    hq = hk * group
    reqs = list(reversed(range(len(held))))
    cu = np.concatenate([[0], np.cumsum([new[r] for r in reqs])])
    tot = int(cu[-1])
    q, qs = c.queries(tot + 2, hq, pad=24)
    scale = -0.2 if case == 3 else dim ** -0.5
    out = torch.full((tot + 2, hq * dim + 8), 7.0, dtype=c.dt, device="cuda")
    lse = torch.full((tot + 2, hq), 7.0, device="cuda")
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale, q_stride_bytes=qs, out_stride_bytes=(hq * dim + 8) * 2)
    ws, size = c.workspace(desc, len(reqs))
    for _ in range(2):
        c.ctx.attn_prompt(c.layer, desc, _i32(reqs), len(reqs), _i32(cu), tot + 2, q, out, lse, ws, size)
    got = out[:, :hq * dim].reshape(tot + 2, hq, dim)
    for i, r in enumerate(reqs):
        a, b = cu[i], cu[i + 1]
        if a < b:
            want, want_lse = _exact(q[a:b], c.rows[r], scale, held[r] - new[r])
            _check(got[a:b], lse[a:b], want, want_lse, f"slot {r}")
    assert (out[tot:] == 7).all() and (lse[tot:] == 7).all() and (out[:, hq * dim:] == 7).all()
    assert c.ctx.stats()["error_count"] == 0
    c.ctx.close()
