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


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1025, 1300])
def test_decode_of_long_lists(n):
    """Lists that are planned by a kernel of their own, with slots that hold nothing in between and a prefix or none."""
    import torch
    from paper_2605_22416_b200 import binding as B
    held = [3, 20, 65, 1]
    c = Cache(held + [0] * n, 2, 64, 16, "bfloat16", seed=3)
    hq, scale = 8, 0.125
    rng = np.random.default_rng(n)
    reqs = rng.integers(0, 4, n)
    reqs[rng.integers(0, n, 5)] = 900
    bad = int((reqs == 900).sum())
    q, _ = c.queries(n, hq)
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale)
    ws, size = c.workspace(desc, n)
    for prefix in (NONE, 2):
        out, lse = torch.full((n, hq, 64), 7.0, dtype=c.dt, device="cuda"), torch.full((n, hq), 7.0, device="cuda")
        before = c.ctx.stats()["error_count"]
        c.ctx.attn_decode(c.layer, desc, _i32(reqs), n, prefix, q, out, lse, ws, size)
        assert c.ctx.stats()["error_count"] - before == bad
        for r in range(4):
            at = torch.from_numpy(np.nonzero(reqs == r)[0]).cuda()
            kv = c.rows[r] if prefix == NONE else torch.cat([c.rows[prefix], c.rows[r]], 1)
            L = kv.shape[1]
            want, want_lse = zip(*(_exact(q[i:i + 1], kv, scale, L - 1) for i in at[:40].tolist()))
            _check(out[at[:40]], lse[at[:40]], torch.cat(want), torch.cat(want_lse), f"slot {r}, prefix {prefix}")
        gone = torch.from_numpy(reqs == 900).cuda()
        assert (out[gone] == 7).all() and (lse[gone] == 7).all()
    c.ctx.close()


@pytest.mark.gpu
def test_prompt_of_many_requests():
    """Lists beyond 32 entries (planned by a kernel of their own), among them empty ones, over splits of the tokens or none."""
    import torch
    from paper_2605_22416_b200 import binding as B
    rng = np.random.default_rng(5)
    held = rng.integers(1, 200, 70).tolist()
    c = Cache(held, 4, 128, 16, "float16", seed=4)
    for hq, most in ((16, 200), (4, 3)):
        new = [int(min(h, rng.integers(0, most))) for h in held]
        cu = np.concatenate([[0], np.cumsum(new)])
        tot = int(cu[-1])
        q, _ = c.queries(tot, hq)
        out, lse = torch.zeros(tot, hq, 128, dtype=c.dt, device="cuda"), torch.zeros(tot, hq, device="cuda")
        desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=0.1)
        ws, size = c.workspace(desc, 70)
        c.ctx.attn_prompt(c.layer, desc, _i32(range(70)), 70, _i32(cu), tot, q, out, lse, ws, size)
        for r in range(70):
            a, b = cu[r], cu[r + 1]
            if a < b:
                want, want_lse = _exact(q[a:b], c.rows[r], 0.1, held[r] - new[r])
                _check(out[a:b], lse[a:b], want, want_lse, f"slot {r}")
    assert c.ctx.stats()["error_count"] == 0
    c.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("total", [6, 700, 9000])
def test_buffers_larger_than_the_rows_in_them(total):
    """A padded batch: far more rows in the buffers than the requests can hold tokens, at widths where the tokens are split
    over the SMs and where they are not; nothing outside the workspace is written."""
    import torch
    from paper_2605_22416_b200 import binding as B
    c = Cache([300, 6], 1, 64, 16, "bfloat16", seed=12)
    desc = B.attn_desc(q_heads=4, dtype=c.dt, scale=0.125)
    size = c.ctx.attn_workspace_bytes(desc, 2)
    ws = torch.full((size + (1 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
    q, _ = c.queries(total, 4)
    out, lse = torch.full((total, 4, 64), 7.0, dtype=c.dt, device="cuda"), torch.full((total, 4), 7.0, device="cuda")
    c.ctx.attn_prompt(c.layer, desc, _i32([0, 1]), 2, _i32([0, 2, 6]), total, q, out, lse, ws, size)
    c.ctx.attn_prompt(c.layer, desc, _i32([0, 1]), 2, _i32([0, 0, 0]), 0, None, None, None, ws, size)      # no rows, no buffers
    assert c.ctx.stats()["error_count"] == 0
    for r, a, b in ((0, 0, 2), (1, 2, 6)):
        want, want_lse = _exact(q[a:b], c.rows[r], 0.125, [300, 6][r] - (b - a))
        _check(out[a:b], lse[a:b], want, want_lse, f"slot {r}")
    assert (out[6:] == 7).all() and (lse[6:] == 7).all() and (ws[size:] == 0x5A).all()
    c.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("lists", ["short", "long"])
def test_bad_items_are_skipped(lists):
    import torch
    from paper_2605_22416_b200 import binding as B
    held = [40, 7, 100, 33] + [5] * 40
    c = Cache(held, 2, 128, 16, "bfloat16", seed=6)
    hq, dim, scale = 4, 128, 0.1
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale)
    # fine, more rows than held, empty slot, out of range, offsets that run backwards, fine, past the buffers
    reqs, cu = [0, 1, 45, 0xFFFFFFF0, 2, 3, 2], [0, 10, 18, 20, 22, 12, 25, 61]
    good = {0: (0, 10), 5: (12, 25)}
    if lists == "long":
        reqs, cu = reqs + list(range(4, 44)), cu + [25] * 40
    bad = len(reqs) - 2 - (0 if lists == "short" else 39)        # the first of the long tail runs backwards too
    n, tot = len(reqs), 60
    q, _ = c.queries(tot, hq)
    ws, size = c.workspace(desc, n)
    out, lse = torch.full((tot, hq, dim), 7.0, dtype=c.dt, device="cuda"), torch.full((tot, hq), 7.0, device="cuda")
    c.ctx.attn_prompt(c.layer, desc, _i32(reqs), n, _i32(cu), tot, q, out, lse, ws, size)
    s = c.ctx.stats()
    assert s["error_count"] == bad and s["error_code"] == 2
    touched = torch.zeros(tot, dtype=torch.bool)
    for i, (a, b) in good.items():
        want, want_lse = _exact(q[a:b], c.rows[reqs[i]], scale, held[reqs[i]] - (b - a))
        _check(out[a:b], lse[a:b], want, want_lse, f"entry {i}")
        touched[a:b] = True
    assert (out[~touched.cuda()] == 7).all() and (lse[~touched.cuda()] == 7).all()
    c.ctx.clear_error()
    # single tokens: an empty slot, one out of range; then a prefix that holds nothing
    reqs = [0, 45, 3, 0xFFFFFFFE]
    out, lse = torch.full((4, hq, dim), 7.0, dtype=c.dt, device="cuda"), torch.full((4, hq), 7.0, device="cuda")
    c.ctx.attn_decode(c.layer, desc, _i32(reqs), 4, NONE, q, out, lse, ws, size)
    assert c.ctx.stats()["error_count"] == 2
    for i in (0, 2):
        want, want_lse = _exact(q[i:i + 1], c.rows[reqs[i]], scale, held[reqs[i]] - 1)
        _check(out[i:i + 1], lse[i:i + 1], want, want_lse, f"entry {i}")
    assert (out[[1, 3]] == 7).all() and (lse[[1, 3]] == 7).all()
    for prefix in (45, 0x7FFFFFF0):
        out.fill_(7)
        c.ctx.clear_error()
        c.ctx.attn_decode(c.layer, desc, _i32(reqs), 4, prefix, q, out, lse, ws, size)
        assert c.ctx.stats()["error_count"] == 4 and (out == 7).all()
    c.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_large_scores_and_zero_scale(dtype):
    """Scores of several hundred, where the running maximum moves from round to round, and a scale of 0 (plain averages)."""
    import torch
    from paper_2605_22416_b200 import binding as B
    held = [700, 1500]
    c = Cache(held, 2, 128, 16, dtype, seed=8)
    # keys that grow along the chain: each round's maximum passes the last one's
    for r, h in enumerate(held):
        kv = c.rows[r].float()
        kv[0] *= torch.linspace(0.02, 4.0, h, device="cuda")[:, None, None]
        c.rows[r] = kv.to(c.dt)
        c.ctx.scatter_kv(c.layer, _i32([r]), None, 1, c.rows[r][0].contiguous(), c.rows[r][1].contiguous())
    hq = 8
    for scale in (1.0, 0.0):
        desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale)
        ws, size = c.workspace(desc, 2)
        cu = [0, 700, 1500]
        q, _ = c.queries(1500, hq, scale=3.0)
        out, lse = torch.zeros(1500, hq, 128, dtype=c.dt, device="cuda"), torch.zeros(1500, hq, device="cuda")
        c.ctx.attn_prompt(c.layer, desc, _i32([0, 1]), 2, _i32(cu), 1500, q, out, lse, ws, size)
        # 32-bit scores of a few hundred are themselves rounded by 2^-15: that moves weights by as much
        slack = 2.0 ** -12 if scale else 0.0
        for r, (a, b) in enumerate(((0, 700), (700, 1500))):
            want, want_lse = _exact(q[a:b], c.rows[r], scale, held[r] - (b - a))
            err = float((out[a:b].double() - want).norm() / want.norm())
            assert err <= 3 * torch.finfo(c.dt).eps / 2 + slack
            assert float((lse[a:b].double() - want_lse).abs().max()) <= 2.0 ** -18 + 2.0 ** -20 * float(want_lse.abs().max())
        out, lse = torch.zeros(2, hq, 128, dtype=c.dt, device="cuda"), torch.zeros(2, hq, device="cuda")
        c.ctx.attn_decode(c.layer, desc, _i32([0, 1]), 2, NONE, q, out, lse, ws, size)
        for r in range(2):
            want, _ = _exact(q[r:r + 1], c.rows[r], scale, held[r] - 1)
            assert float((out[r:r + 1].double() - want).norm() / want.norm()) <= 3 * torch.finfo(c.dt).eps / 2 + slack
    c.ctx.close()


@pytest.mark.gpu
def test_nan_in_a_chain_stays_with_the_rows_that_see_it():
    import torch
    from paper_2605_22416_b200 import binding as B
    c = Cache([300, 50], 2, 64, 16, "bfloat16", seed=9)
    kv = c.rows[0].clone()
    kv[0, 200, 1, 5] = math.nan                   # a key of head 1
    c.ctx.scatter_kv(c.layer, _i32([0]), None, 1, kv[0].contiguous(), kv[1].contiguous())
    desc = B.attn_desc(q_heads=4, dtype=c.dt, scale=0.125)
    ws, size = c.workspace(desc, 2)
    q, _ = c.queries(350, 4)
    out = torch.zeros(350, 4, 64, dtype=c.dt, device="cuda")
    c.ctx.attn_prompt(c.layer, desc, _i32([0, 1]), 2, _i32([0, 300, 350]), 350, q, out, None, ws, size)
    nan = out.isnan().all(-1)
    assert nan[200:300, 2:].all() and not nan[:200].any() and not nan[:, :2].any() and not nan[300:].any()
    assert torch.isfinite(out[:200]).all() and torch.isfinite(out[300:]).all()
    c.ctx.close()


@pytest.mark.gpu
def test_graph_replay_other_stream_and_shared_workspace():
    """A captured step (prompt, decode, decode behind a prefix, one after the other on one workspace) replays bit for bit, on
    another stream too, and sees tokens that were appended in between."""
    import torch
    from paper_2605_22416_b200 import binding as B
    held = [90, 300, 17, 700]
    c = Cache(held, 4, 128, 16, "bfloat16", seed=11)
    hq, dim, scale = 8, 128, 0.09
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale)
    ws, size = c.workspace(desc, 3)
    q, _ = c.queries(60, hq)
    cu, reqs = _i32([0, 30, 50, 60]), _i32([0, 1, 2])
    bufs = [torch.zeros(60, hq, dim, dtype=c.dt, device="cuda") for _ in range(3)]
    c.ctx.attn_decode(c.layer, desc, 0, 0, NONE, 0, 0, None, ws, size)
    c.ctx.attn_prompt(c.layer, desc, 0, 0, 0, 0, 0, 0, None, ws, size)

    def step():
        c.ctx.attn_prompt(c.layer, desc, reqs, 3, cu, 60, q, bufs[0], None, ws, size)
        c.ctx.attn_decode(c.layer, desc, reqs, 3, NONE, q, bufs[1], None, ws, size)
        c.ctx.attn_decode(c.layer, desc, reqs, 3, 3, q, bufs[2], None, ws, size)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    want = [b.clone() for b in bufs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        for b in bufs:
            b.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bufs, want))
    # three more tokens for slot 0: the same graph reads the longer chain
    st = np.zeros(1, np.uint32)
    c.ctx.step_host(W.make_ops(W.OP_EXTEND, [0], 3), 1, st)
    assert st[0] == 0
    kv = torch.randn(2, 3, 4, dim, device="cuda", generator=c.gen).to(c.dt)
    c.ctx.scatter_kv(c.layer, _i32([0]), _i32([90]), 1, kv[0].contiguous(), kv[1].contiguous())
    c.rows[0] = torch.cat([c.rows[0], kv], 1)
    graph.replay()
    torch.cuda.synchronize()
    for buf, a, b, past, pre in ((bufs[0], 0, 30, 63, None), (bufs[1], 0, 1, 92, None), (bufs[2], 0, 1, 92 + 700, 3)):
        kv = c.rows[0] if pre is None else torch.cat([c.rows[pre], c.rows[0]], 1)
        w, l = _exact(q[a:b], kv, scale, past)
        _check(buf[a:b], l.float(), w, l, "after three more tokens")
    c.ctx.close()


@pytest.mark.gpu
def test_run_of_both_caches_in_a_step():
    """The calls as an engine makes them: admit, write the prompt's rows, prompt attention and recurrence, then single-token
    steps that extend the chain, write one row and attend; a migration of capacity in between moves pages and blocks."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt, hk, hq, dim, heads, dk, dv = torch.bfloat16, 2, 8, 64, 4, 16, 64
    m = SimpleNamespace(n_attn_layers=2, n_ssm_layers=2, page_tokens=16, kv_heads=hk, head_dim=dim, kv_elem_bytes=2,
                        ssm_state_elems=heads * dk * dv, ssm_conv_elems=64, ssm_elem_bytes=4)
    u_kv, u_ssm = 2 * 2 * 16 * hk * dim * 2, 4 * (heads * dk * dv + 64)
    pool = 17 * u_kv + 16 * u_ssm + 256
    ctx = B.Context(m, pool, (16 * u_ssm + 128) / pool, 12, max_requests=8, max_pages=40, min_rebalance_interval_ops=1)
    gen = torch.Generator("cuda").manual_seed(2)
    lens, st = [50, 33, 80], np.zeros(3, np.uint32)
    reqs, n = [4, 0, 6], 3
    # others come first and leave again, so that these requests hold the blocks that a migration takes
    more = np.zeros(5, np.uint32)
    ctx.step_host(W.make_ops(W.OP_ADMIT, [1, 2, 3, 5, 7], 1), 5, more)
    ctx.step_host(W.make_ops(W.OP_ADMIT, reqs, lens), 3, st)
    assert (st == 0).all() and (more == 0).all()
    ctx.step_host(W.make_ops(W.OP_FINISH, [1, 2, 3, 5, 7], 0), 5, more)
    tot, cu = sum(lens), np.concatenate([[0], np.cumsum(lens)])
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    ad = B.attn_desc(q_heads=hq, dtype=dt, scale=dim ** -0.5)
    sd = B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=dt)
    ws = torch.empty(ctx.attn_workspace_bytes(ad, 8), dtype=torch.uint8, device="cuda")
    k, v, q = rnd(tot, hk, dim).to(dt), rnd(tot, hk, dim).to(dt), rnd(tot, hq, dim).to(dt)
    sq, sk, sv, sg = (rnd(tot, 1, dk) * 0.3).to(dt), rnd(tot, 1, dk).to(dt), rnd(tot, heads, dv).to(dt), -torch.rand(tot, heads, device="cuda", generator=gen)
    out, sout = torch.zeros_like(q), torch.zeros_like(sv)
    ctx.scatter_kv(1, _i32(reqs), None, n, k, v)
    ctx.attn_prompt(1, ad, _i32(reqs), n, _i32(cu), tot, q, out, None, ws, ws.numel())
    ctx.ssm_prompt(1, sd, _i32(reqs), n, _i32(cu), tot, None, sq, sk, sv, sg, sout)
    chain = [torch.stack([k[a:b], v[a:b]]) for a, b in zip(cu, cu[1:])]
    state = []
    for i, (a, b) in enumerate(zip(cu, cu[1:])):
        w, l = _exact(q[a:b], chain[i], dim ** -0.5, 0)
        _check(out[a:b], l.float(), w, l, f"prompt {i}")
        S = torch.zeros(heads, dv, dk, dtype=torch.float64, device="cuda")
        for t in range(a, b):
            S = S * sg[t].double().exp()[:, None, None] + sv[t].double()[:, :, None] * sk[t].double()[:, None, :]
        state.append(S)
    for step in range(6):
        grow = 30 if step == 3 else 1                # one step appends a turn: KV pages run out and SSM capacity moves over
        ctx.step_host(W.make_ops(W.OP_EXTEND, reqs, grow), 3, st)
        assert (st == 0).all()
        k, v, q = rnd(3 * grow, hk, dim).to(dt), rnd(3 * grow, hk, dim).to(dt), rnd(3, hq, dim).to(dt)
        held = [c.shape[1] for c in chain]
        ctx.scatter_kv(1, _i32(reqs), _i32(held), n, k, v)
        chain = [torch.cat([c, torch.stack([k[i * grow:(i + 1) * grow], v[i * grow:(i + 1) * grow]])], 1) for i, c in enumerate(chain)]
        sq, sk, sv, sg = (rnd(3, 1, dk) * 0.3).to(dt), rnd(3, 1, dk).to(dt), rnd(3, heads, dv).to(dt), -torch.rand(3, heads, device="cuda", generator=gen)
        out, sout = torch.zeros_like(q), torch.zeros_like(sv)
        ctx.attn_decode(1, ad, _i32(reqs), n, NONE, q, out, None, ws, ws.numel())
        ctx.ssm_step(1, sd, _i32(reqs), n, sq, sk, sv, sg, sout)
        for i in range(3):
            w, l = _exact(q[i:i + 1], chain[i], dim ** -0.5, chain[i].shape[1] - 1)
            _check(out[i:i + 1], l.float(), w, l, f"step {step}, request {i}")
            state[i] = state[i] * sg[i].double().exp()[:, None, None] + sv[i].double()[:, :, None] * sk[i].double()[:, None, :]
            o = (state[i] * sq[i].double()).sum(-1)
            assert float((sout[i].double() - o).norm() / o.norm()) <= torch.finfo(dt).eps / 2
    s = ctx.stats()
    assert s["error_count"] == 0 and s["n_rebalance"] > 0 and s["relocated_blocks"] > 0, s
    got = torch.empty(3, heads, dv, dk, device="cuda")
    ctx.gather_ssm(1, _i32(reqs), 3, got, torch.empty(3, 64, device="cuda"))
    for i in range(3):
        assert float((got[i].double() - state[i]).norm() / state[i].norm()) <= 2.0 ** -18
    ctx.close()


def test_refusals_on_the_host():
    """Arguments are checked before anything is launched; this part needs no context."""
    import ctypes
    import torch
    from paper_2605_22416_b200 import binding as B
    with pytest.raises(B.AvmpError):
        B.attn_desc(q_heads=1, dtype=torch.float32, scale=1.0)
    d = B.attn_desc(q_heads=4, dtype=torch.float16, scale=1.0)
    assert B.lib.avmp_attn_workspace_bytes(None, ctypes.byref(d), 1) == 0
    assert B.lib.avmp_attn_decode(None, 0, ctypes.byref(d), None, 1, 0, None, None, None, None, 0, None) == B.AVMP_EINVAL
    assert B.lib.avmp_attn_prompt(None, 0, ctypes.byref(d), None, 1, None, 0, None, None, None, None, 0, None) == B.AVMP_EINVAL


@pytest.mark.gpu
def test_refusals():
    import torch
    from paper_2605_22416_b200 import binding as B
    c = Cache([20, 3], 2, 64, 16, "bfloat16", seed=1)
    x = torch.zeros(1 << 16, dtype=torch.bfloat16, device="cuda")
    f = torch.zeros(64, device="cuda")
    ok = dict(q_heads=4, dtype=torch.bfloat16, scale=0.1)
    good = B.attn_desc(**ok)
    ws, size = c.workspace(good, 5)
    reqs, cu = _i32([0]), _i32([0, 1])

    def decode(layer=0, n=1, q=x, o=x, lse=None, w=ws, ws_bytes=size, reqs=reqs, **kw):
        c.ctx.attn_decode(layer, B.attn_desc(**{**ok, **kw}), reqs, n, NONE, q, o, lse, w, ws_bytes)

    def prompt(layer=0, n=1, q=x, o=x, lse=None, w=ws, ws_bytes=size, reqs=reqs, cu=cu, total=1, **kw):
        c.ctx.attn_prompt(layer, B.attn_desc(**{**ok, **kw}), reqs, n, cu, total, q, o, lse, w, ws_bytes)

    bad = [dict(layer=3), dict(n=6), dict(q_heads=3), dict(q_heads=0), dict(q_heads=130), dict(scale=math.inf), dict(scale=math.nan),
           dict(q_stride_bytes=24), dict(out_stride_bytes=256), dict(q=x.data_ptr() + 2), dict(q=None), dict(o=x.data_ptr() + 8),
           dict(o=None), dict(lse=f.data_ptr() + 2), dict(w=None), dict(w=ws.data_ptr() + 8), dict(reqs=None)]
    for kw in bad:
        for call in (decode, prompt):
            with pytest.raises(B.AvmpError, match="invalid argument"):
                call(**kw)
    for call in (decode, prompt):
        with pytest.raises(B.AvmpError, match="workspace too small"):
            call(ws_bytes=c.ctx.attn_workspace_bytes(good, 1) - 1)
    for kw in (dict(cu=None), dict(total=1 << 30)):
        with pytest.raises(B.AvmpError, match="invalid argument"):
            prompt(**kw)
    wrong = B.attn_desc(**ok)
    wrong.type = 2
    assert c.ctx.attn_workspace_bytes(wrong, 1) == 0 and c.ctx.attn_workspace_bytes(good, 6) == 0
    assert c.ctx.stats()["error_count"] == 0
    c.ctx.close()
    for dim, page, elem in ((96, 16, 2), (64, 12, 2), (64, 16, 4)):      # shapes that the kernels do not have
        m = SimpleNamespace(n_attn_layers=1, n_ssm_layers=1, page_tokens=page, kv_heads=2, head_dim=dim, kv_elem_bytes=elem,
                            ssm_state_elems=64, ssm_conv_elems=4, ssm_elem_bytes=4)
        ctx = B.Context(m, 1 << 20, 0.1, 1, max_requests=4, max_pages=4)
        assert ctx.attn_workspace_bytes(good, 1) == 0
        with pytest.raises(B.AvmpError, match="invalid argument"):
            ctx.attn_decode(0, good, reqs, 1, NONE, x, x, None, ws, size)
        ctx.close()
