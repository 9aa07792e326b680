"""Norms, rotation and cache writes of new rows (avmp_attn_rows_*) and attention through a window (avmp_attn_window_*) against their
formulas in 64 bits, and a run of all calls of a hybrid step together.

Tolerances.  Rows: the norm's factor is off by a few 2^-23 (mean of squares, reciprocal root), a rotated column by 2^-21 of its
pair's magnitudes (sine and cosine, two products), then one rounding to 16 bits; fp16 results below its normal range by 2^-25 at most.  Values are
copied: equal.  Attention: as derived in test_attn_ops.py.
"""
from __future__ import annotations

import math

import numpy as np
import pytest

from test_attn_ops import Cache, _check, _i32
from test_conv_scan import _conv_exact, _scan_exact
from types import SimpleNamespace

from paper_2605_22416_b200 import workloads as W


# ---------------------------------------------------------------- rows
def _rotated(x, weight, eps, place, freq, neighbours):
    """x [L, heads, dim] -> the formula in 64 bits, and its bound."""
    import torch
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    size = x.abs()
    if freq is not None:
        half = freq.numel()
        i = torch.arange(half, device="cuda")
        p, q = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
        t = place.double()[:, None] * freq.double()
        c, s = t.cos()[:, None], t.sin()[:, None]
        y = x.clone()
        y[..., p], y[..., q] = x[..., p] * c - x[..., q] * s, x[..., q] * c + x[..., p] * s
        size = size.clone()
        size[..., p] = size[..., q] = x[..., p].abs() + x[..., q].abs()
        x = y
    return x, size * 2.0 ** -21


def _near(got, want, bound, what):
    import torch
    assert torch.isfinite(got).all(), what
    off = (got.double() - want).abs() - bound - (want.abs() + bound) * (torch.finfo(got.dtype).eps / 2) - 2.0 ** -25
    assert float(off.max()) <= 0, f"{what}: {float(off.max()):.3g} over the bound"


def _cached(c, r):
    """K and V of a slot's chain, [held, kv_heads, dim] each."""
    import torch
    k, v = (torch.empty(c.held[r], c.kv_heads, c.dim, dtype=c.dt, device="cuda") for _ in range(2))
    c.ctx.gather_kv(c.layer, _i32([r]), 1, k, v, c.held[r], torch.empty(2, dtype=torch.int32, device="cuda"))
    return k, v


ROWS = [
    # held, new, kv_heads, group, dim, page, rotary, neighbours, norm, positions
    ([1], [1], 1, 1, 64, 16, 64, False, True, False),
    ([16, 17, 40, 200], [16, 1, 0, 130], 8, 4, 128, 16, 128, False, True, False),
    ([70, 9, 33], [3, 9, 33], 2, 3, 128, 32, 32, True, True, True),
    ([100, 2], [64, 2], 4, 1, 64, 8, 16, True, False, False),
    ([65, 30], [65, 7], 3, 5, 64, 24, 40, False, True, True),
    ([50], [20], 2, 2, 128, 16, 0, False, True, False),
    ([300, 1, 77], [299, 1, 5], 1, 7, 128, 64, 128, True, False, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(ROWS)))
def test_rows(dtype, case):
    import torch
    from paper_2605_22416_b200 import binding as B
    held, new, hk, group, dim, page, rotary, neighbours, norm, with_pos = ROWS[case]
    c = Cache(held, hk, dim, page, dtype, seed=case)
    hq, tot, gen = hk * group, sum(new), c.gen
    width = (hq + 2 * hk) * dim
    qkv = (torch.randn(tot, width + 16, device="cuda", generator=gen) * 2).to(c.dt)
    q, k, v = (x.unflatten(1, (-1, dim)) for x in qkv[:, :width].split([hq * dim, hk * dim, hk * dim], 1))
    wq, wk = ((1 + 0.3 * torch.randn(dim, device="cuda", generator=gen)) if norm else None for _ in range(2))
    freq = (10000.0 ** (-torch.arange(rotary // 2, device="cuda") / (rotary // 2))).float() if rotary else None
    cu = np.concatenate([[0], np.cumsum(new)])
    place = np.concatenate([np.arange(h - a, h) for h, a in zip(held, new)])
    if with_pos:
        place = np.random.default_rng(case).integers(0, 1 << 24, tot)
    out = torch.full((tot + 1, hq * dim + 8), 7.0, dtype=c.dt, device="cuda")
    stride = (width + 16) * 2
    desc = B.rows_desc(q_heads=hq, rotary_dim=rotary, neighbours=neighbours, eps=1e-5, dtype=c.dt, q_stride_bytes=stride, k_stride_bytes=stride,
                       v_stride_bytes=stride, out_stride_bytes=(hq * dim + 8) * 2)
    n, reqs = len(held), list(range(len(held)))
    pos = _i32(place) if with_pos else None
    c.ctx.attn_rows_prompt(c.layer, desc, _i32(reqs), n, _i32(cu), tot, pos, q, k, v, wq, wk, freq, out)
    at = torch.tensor(place, device="cuda")
    want_q, bound_q = _rotated(q, wq, 1e-5, at, freq, neighbours)
    want_k, bound_k = _rotated(k, wk, 1e-5, at, freq, neighbours)
    _near(out[:tot, :hq * dim].unflatten(1, (hq, dim)), want_q, bound_q, "queries")
    assert (out[:, hq * dim:] == 7).all() and (out[tot:] == 7).all()
    for r in reqs:
        kk, vv = _cached(c, r)
        old, sl = held[r] - new[r], slice(cu[r], cu[r + 1])
        assert torch.equal(kk[:old], c.rows[r][0][:old]) and torch.equal(vv[:old], c.rows[r][1][:old])
        if new[r]:
            _near(kk[old:], want_k[sl], bound_k[sl], f"keys of {r}")
            assert torch.equal(vv[old:], v[sl])
    # one token per request is the same thing
    out1 = torch.empty(n, hq, dim, dtype=c.dt, device="cuda")
    desc1 = B.rows_desc(q_heads=hq, rotary_dim=rotary, neighbours=neighbours, eps=1e-5, dtype=c.dt)
    one = [torch.randn(n, h, dim, device="cuda", generator=gen).to(c.dt) for h in (hq, hk, hk)]
    at = torch.tensor(np.asarray(held) - 1, device="cuda") if not with_pos else torch.arange(n, device="cuda") * 1000
    c.ctx.attn_rows_step(c.layer, desc1, _i32(reqs), n, _i32(at.cpu().numpy()) if with_pos else None, *one, wq, wk, freq, out1)
    _near(out1, *_rotated(one[0], wq, 1e-5, at, freq, neighbours), "queries, single tokens")
    want_k, bound_k = _rotated(one[1], wk, 1e-5, at, freq, neighbours)
    for r in reqs:
        kk, vv = _cached(c, r)
        _near(kk[-1:], want_k[r:r + 1], bound_k[r:r + 1], f"key of {r}")
        assert torch.equal(vv[-1], one[2][r])
    assert c.ctx.stats()["error_count"] == 0
    c.ctx.close()


@pytest.mark.gpu
def test_rows_bad_items_and_refusals():
    import torch
    from paper_2605_22416_b200 import binding as B
    held = [20, 30, 5, 8]
    c = Cache(held, 2, 64, 16, "bfloat16")
    hq, dim = 4, 64
    tot = 60
    q, k, v = (torch.randn(tot, h, dim, device="cuda", generator=c.gen).to(c.dt) for h in (hq, 2, 2))
    freq = torch.rand(32, device="cuda", generator=c.gen)
    out = torch.full((tot, hq, dim), 7.0, dtype=c.dt, device="cuda")
    ok = dict(q_heads=hq, rotary_dim=64, neighbours=False, eps=1e-6, dtype=c.dt)
    desc = B.rows_desc(**ok)
    # named before; empty; out of range; more rows than held tokens; decreasing; past the rows
    reqs, cu = [1, 1, 5, 99, 2, 3, 0], [0, 10, 14, 16, 18, 26, 20, 70]
    c.ctx.attn_rows_prompt(c.layer, desc, _i32(reqs), 7, _i32(cu), tot, None, q, k, v, None, None, freq, out)
    assert c.ctx.stats()["error_count"] == 6
    place = torch.arange(20, 30, device="cuda")
    _near(out[:10], *_rotated(q[:10], None, 0, place, freq, False), "queries")
    assert (out[10:] == 7).all()
    for r in (0, 2, 3):
        kk, vv = _cached(c, r)
        assert torch.equal(kk, c.rows[r][0]) and torch.equal(vv, c.rows[r][1])
    kk, vv = _cached(c, 1)
    assert torch.equal(vv[20:], v[:10]) and torch.equal(kk[:20], c.rows[1][0][:20])
    c.ctx.clear_error()
    # frequencies and weights are what they are: a row of zeros with eps 0 has no direction, and says so
    c.ctx.attn_rows_step(c.layer, B.rows_desc(**{**ok, "eps": 0.0}), _i32([0, 5, 0]), 3, None, torch.zeros_like(q), k, v, freq.repeat(2), None, freq, out)
    assert c.ctx.stats()["error_count"] == 2 and torch.isnan(out[0]).all()

    def call(layer=1, n=1, qq=q, kk=k, fr=freq, o=out, **kw):
        d = B.rows_desc(**{**ok, **kw})
        c.ctx.attn_rows_prompt(layer, d, _i32([0]), n, _i32([0, 1]), tot, None, qq, kk, v, None, None, fr, o)

    call()
    for bad in (dict(layer=3), dict(n=99), dict(q_heads=0), dict(rotary_dim=4), dict(rotary_dim=72), dict(eps=-1.0), dict(eps=math.nan), dict(fr=None),
                dict(qq=None), dict(qq=q.view(-1)[4:]), dict(kk=None), dict(o=None), dict(q_stride_bytes=16), dict(v_stride_bytes=100)):
        with pytest.raises(B.AvmpError):
            call(**bad)
    with pytest.raises(B.AvmpError):
        B.rows_desc(**{**ok, "dtype": torch.float32})
    c.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("neighbours", [False, True])
def test_rows_infinities_stay_in_their_pair(neighbours):
    """Without norms: an infinity in a rotated column is seen in its pair, one in a column that is not rotated in that column alone."""
    import torch
    from paper_2605_22416_b200 import binding as B
    c = Cache([3], 2, 64, 16, "bfloat16")
    q, k, v = (torch.randn(3, h, 64, device="cuda", generator=c.gen).to(c.dt) for h in (4, 2, 2))
    freq = torch.rand(16, device="cuda", generator=c.gen) + 0.1
    out = torch.empty(3, 4, 64, dtype=c.dt, device="cuda")
    desc = B.rows_desc(q_heads=4, rotary_dim=32, neighbours=neighbours, eps=0.0, dtype=c.dt)
    bad = {(1, 0, 3), (2, 1, 40), (2, 3, 63)}
    for t, h, col in bad:
        q[t, h, col] = math.inf
    c.ctx.attn_rows_prompt(c.layer, desc, _i32([0]), 1, _i32([0, 3]), 3, None, q, k, v, None, None, freq, out)
    hit = torch.zeros(3, 4, 64, dtype=torch.bool, device="cuda")
    hit[1, 0, [2, 3] if neighbours else [3, 19]] = True
    hit[2, 1, 40] = hit[2, 3, 63] = True
    assert torch.equal(~torch.isfinite(out), hit) and out[2, 1, 40] == math.inf
    want, bound = _rotated(torch.where(hit, 0, q), None, 0, torch.arange(3, device="cuda"), freq, neighbours)
    _near(torch.where(hit, 0, out), torch.where(hit, 0, want), bound, "the others")
    c.ctx.close()


# ---------------------------------------------------------------- window
def _exact(q, kv, scale, past, window, sinks):
    import torch
    rep = q.shape[1] // kv.shape[2]
    K, V = (x.double().repeat_interleave(rep, 1) for x in kv)
    z = torch.einsum("ihd,jhd->hij", q.double(), K) * scale
    j, i = torch.arange(kv.shape[1], device="cuda")[None], (torch.arange(q.shape[0], device="cuda") + past)[:, None]
    z.masked_fill_((j > i) | ((j <= i - window) & (j >= sinks)), -math.inf)
    lse = torch.logsumexp(z, -1)
    return torch.einsum("hij,jhd->ihd", (z - lse[..., None]).exp(), V), lse.transpose(0, 1)


WINDOWS = [(1, 0), (1, 1), (7, 3), (16, 16), (64, 4), (129, 0), (100, 200), (300, 129), (10 ** 6, 5), (0xFFFFFFFF, 0xFFFFFFFF)]
DECODE = [
    # held, kv_heads, group, dim, page
    ([1, 2, 600, 33], 1, 1, 64, 16),
    ([16, 17, 15, 1, 900], 8, 4, 128, 16),
    ([129, 64, 3000], 4, 8, 64, 32),
    ([500, 31, 8, 9], 1, 40, 128, 16),
    ([250, 7], 5, 3, 64, 24),
    ([90, 1, 400], 16, 2, 128, 8),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(DECODE)))
def test_window_decode(dtype, case):
    """What no row sees is NaN in the cache, keys and values."""
    import torch
    from paper_2605_22416_b200 import binding as B
    held, hk, group, dim, page = DECODE[case]
    for window, sinks in WINDOWS:
        c = Cache(held, hk, dim, page, dtype, seed=case)
        n, hq, scale = len(held), hk * group, dim ** -0.5
        q, qs = c.queries(n, hq, pad=8)
        desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale, q_stride_bytes=qs)
        out, lse = torch.full((n, hq, dim), 7.0, dtype=c.dt, device="cuda"), torch.empty(n, hq, device="cuda")
        ws, size = c.workspace(desc, n)
        want = []
        for r in range(n):
            want.append(_exact(q[r:r + 1], c.rows[r], scale, held[r] - 1, window, sinks))
            j = torch.arange(held[r], device="cuda")
            hidden = (j < held[r] - min(window, held[r])) & (j >= min(sinks, 1 << 30))
            kv = c.rows[r].clone()
            kv[:, hidden] = math.nan
            c.ctx.scatter_kv(c.layer, _i32([r]), None, 1, kv[0].contiguous(), kv[1].contiguous())
        c.ctx.attn_window_decode(c.layer, desc, window, sinks, _i32(range(n)), n, q, out, lse, ws, size)
        _check(out, lse, torch.cat([w[0] for w in want]), torch.cat([w[1] for w in want]), f"window {window}, sinks {sinks}")
        assert c.ctx.stats()["error_count"] == 0
        c.ctx.close()


PROMPT = [
    # held, new, kv_heads, group, dim, page
    ([1], [1], 1, 1, 64, 16),
    ([300, 17, 40, 700], [300, 1, 12, 130], 2, 4, 128, 16),
    ([513, 64], [200, 64], 4, 1, 64, 32),
    ([1500], [1400], 1, 8, 128, 64),
    ([600, 9], [500, 0], 1, 3, 128, 8),
    ([700] * 40, [30] * 40, 1, 2, 64, 16),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(PROMPT)))
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_window_prompt(dtype, case, window, sinks):
    import torch
    from paper_2605_22416_b200 import binding as B
    held, new, hk, group, dim, page = PROMPT[case]
    c = Cache(held, hk, dim, page, dtype, seed=case)
    n, hq, scale, tot = len(held), hk * group, dim ** -0.5, sum(new)
    q, qs = c.queries(tot, hq, pad=8)
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale, q_stride_bytes=qs)
    out, lse = torch.full((tot + 1, hq, dim), 7.0, dtype=c.dt, device="cuda"), torch.full((tot + 1, hq), 7.0, device="cuda")
    ws, size = c.workspace(desc, n)
    cu = np.concatenate([[0], np.cumsum(new)])
    want = [_exact(q[cu[r]:cu[r + 1]], c.rows[r], scale, held[r] - new[r], window, sinks) for r in range(n) if new[r]]
    for r in range(n):
        j = torch.arange(held[r], device="cuda")
        first = held[r] - new[r]
        hidden = (j < first + 1 - min(window, first + 1)) & (j >= min(sinks, 1 << 30))      # what not even the first row sees
        if hidden.any():
            kv = c.rows[r].clone()
            kv[:, hidden] = math.nan
            c.ctx.scatter_kv(c.layer, _i32([r]), None, 1, kv[0].contiguous(), kv[1].contiguous())
    c.ctx.attn_window_prompt(c.layer, desc, window, sinks, _i32(range(n)), n, _i32(cu), tot, q, out, lse, ws, size)
    _check(out[:tot], lse[:tot], torch.cat([w[0] for w in want]), torch.cat([w[1] for w in want]), "prompt")
    assert (out[tot:] == 7).all() and (lse[tot:] == 7).all() and c.ctx.stats()["error_count"] == 0
    c.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("window,sinks", [(50, 0), (200, 3), (150, 140)])
def test_nonfinite_values_reach_the_rows_that_see_them(dtype, n, window, sinks):
    """NaN and infinities among the values: in every row that sees them, in no other."""
    import torch
    from paper_2605_22416_b200 import binding as B
    held = [420] * n
    c = Cache(held, 1, 64, 16, dtype, seed=n)
    hq, new, scale = 2, 300, 0.125
    q, _ = c.queries(n * new, hq)
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale)
    ws, size = c.workspace(desc, n)
    bad = {0: math.inf, 130: math.nan, 200: -math.inf, 290: math.inf, 419: math.nan}
    out = torch.empty(n * new, hq, 64, dtype=c.dt, device="cuda")
    for r in range(n):
        kv = c.rows[r].clone()
        for t, x in bad.items():
            kv[1, t, 0, t % 64] = x
        c.ctx.scatter_kv(c.layer, _i32([r]), None, 1, kv[0].contiguous(), kv[1].contiguous())
    c.ctx.attn_window_prompt(c.layer, desc, window, sinks, _i32(range(n)), n, _i32(np.arange(n + 1) * new), n * new, q, out, None, ws, size)
    for r in range(0, n, 13):
        o = out[r * new:(r + 1) * new]
        want, _ = _exact(q[r * new:(r + 1) * new], c.rows[r], scale, 120, window, sinks)
        p = torch.arange(120, 420, device="cuda")
        hit = torch.zeros(new, 64, dtype=torch.bool, device="cuda")
        for t in bad:
            hit[:, t % 64] |= (p >= t) & ((t > p - window) | (t < sinks))
        hit = hit[:, None].expand(-1, hq, -1)
        assert torch.equal(torch.isfinite(o), ~hit)
        clean, w = torch.where(hit, 0, o.float()), torch.where(hit, 0, want)
        assert float((clean - w).norm() / w.norm()) <= 3 * torch.finfo(c.dt).eps / 2
    assert c.ctx.stats()["error_count"] == 0
    c.ctx.close()


@pytest.mark.gpu
def test_window_items_and_refusals():
    import torch
    from paper_2605_22416_b200 import binding as B
    c = Cache([40, 25], 2, 64, 16, "bfloat16")
    q, _ = c.queries(40, 4)
    desc = B.attn_desc(q_heads=4, dtype=c.dt, scale=0.125)
    ws, size = c.workspace(desc, 4)
    out = torch.full((40, 4, 64), 7.0, dtype=c.dt, device="cuda")
    c.ctx.attn_window_decode(1, desc, 8, 2, _i32([0, 4, 77, 0]), 4, q, out, None, ws, size)
    assert c.ctx.stats()["error_count"] == 2 and (out[1:3] == 7).all() and (out[4:] == 7).all()
    for row in (0, 3):
        want, _ = _exact(q[row:row + 1], c.rows[0], 0.125, 39, 8, 2)
        assert float((out[row:row + 1].double() - want).norm() / want.norm()) <= 3 * 2.0 ** -8
    out.fill_(7.0)
    c.ctx.attn_window_prompt(1, desc, 8, 2, _i32([1, 4, 0, 1]), 4, _i32([0, 26, 28, 30, 29]), 40, q, out, None, ws, size)
    assert c.ctx.stats()["error_count"] == 5
    want, _ = _exact(q[28:30], c.rows[0], 0.125, 38, 8, 2)
    assert float((out[28:30].double() - want).norm() / want.norm()) <= 3 * 2.0 ** -8 and (out[:28] == 7).all() and (out[30:] == 7).all()
    for bad in (dict(window=0), dict(layer=3), dict(n=9), dict(size=size // 2), dict(ws=None), dict(q=None)):
        a = {**dict(window=8, layer=1, n=2, size=size, ws=ws, q=q), **bad}
        with pytest.raises(B.AvmpError):
            c.ctx.attn_window_decode(a["layer"], desc, a["window"], 2, _i32([0, 1]), a["n"], a["q"], out, None, a["ws"], a["size"])
        with pytest.raises(B.AvmpError):
            c.ctx.attn_window_prompt(a["layer"], desc, a["window"], 2, _i32([0, 1]), a["n"], _i32([0, 1, 2]), 2, a["q"], out, None, a["ws"], a["size"])
    c.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_bounded_waits_of_the_window_calls(call):
    """With any limit a call is either reported or right, bit for bit."""
    import torch
    from paper_2605_22416_b200 import binding as B
    c = Cache([900, 300, 70], 2, 128, 16, "bfloat16")
    q, _ = c.queries(600 if call == "prompt" else 3, 8)
    desc = B.attn_desc(q_heads=8, dtype=c.dt, scale=0.1)
    ws, size = c.workspace(desc, 3)

    def run():
        out = torch.zeros(q.shape, dtype=c.dt, device="cuda")
        if call == "prompt":
            c.ctx.attn_window_prompt(1, desc, 200, 4, _i32([0, 1, 2]), 3, _i32([0, 400, 550, 600]), 600, q, out, None, ws, size)
        else:
            c.ctx.attn_window_decode(1, desc, 200, 4, _i32([0, 1, 2]), 3, q, out, None, ws, size)
        return out

    want = run()
    for ns in (0, 500, 2000, 10000, 100000, 2000000000):
        c.ctx.set_wait_limit(ns)
        out = run()
        s = c.ctx.stats()
        assert s["error_code"] in (0, 4)
        assert s["error_code"] == 4 or torch.equal(out, want)
        c.ctx.clear_error()
    assert torch.equal(out, want)
    c.ctx.close()


# ---------------------------------------------------------------- a hybrid step
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_hybrid_layers_over_a_prompt_and_tokens(dtype):
    """Prompts, then three tokens each in a captured graph, through convolution, scan, rows and window attention, on a side stream.  Each call's
    inputs are the library's own outputs of the call before; its results are compared with the formulas on these."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = getattr(torch, dtype)
    d, ns, w, hk, hq, dim, T = 256, 16, 4, 2, 4, 64, 16
    m = SimpleNamespace(n_attn_layers=1, n_ssm_layers=1, page_tokens=T, kv_heads=hk, head_dim=dim, kv_elem_bytes=2, ssm_state_elems=d * ns,
                        ssm_conv_elems=d * (w - 1), ssm_elem_bytes=4)
    ctx = B.Context(m, 4 << 20, 0.5, 4, max_requests=8, max_pages=32)
    gen = torch.Generator("cuda").manual_seed(5)
    normal = lambda *shape, s=1.0: torch.randn(*shape, device="cuda", generator=gen) * s
    lens, reqs, window, sinks = [90, 1, 300], [4, 1, 6], 64, 3
    st = np.zeros(3, np.uint32)
    ctx.step_host(W.make_ops(W.OP_ADMIT, reqs, lens), 3, st)
    assert (st == 0).all()
    weight, bias, a, skip = normal(d, w, s=0.5), normal(d), -torch.exp(normal(d, ns) * 0.5), normal(d)
    wq, wk = 1 + normal(dim, s=0.1), 1 + normal(dim, s=0.1)
    freq = (10000.0 ** (-torch.arange(dim // 2, device="cuda") / (dim // 2))).float()
    proj = normal(d, d + 2 * ns, s=d ** -0.5).to(dt)
    up = normal(d, (hq + 2 * hk) * dim, s=d ** -0.5).to(dt)
    conv = B.conv_desc(channels=d, width=w, silu=True, dtype=dt, x_stride_bytes=4 * d)
    sb = (d + 2 * ns) * 2
    scan = B.scan_desc(channels=d, groups=1, states=ns, softplus=True, dtype=dt, delta_stride_bytes=sb, z_stride_bytes=4 * d, b_stride_bytes=sb,
                       c_stride_bytes=sb)
    qs = (hq + 2 * hk) * dim * 2
    rows = B.rows_desc(q_heads=hq, rotary_dim=dim, neighbours=False, eps=1e-6, dtype=dt, q_stride_bytes=qs, k_stride_bytes=qs, v_stride_bytes=qs)
    attn = B.attn_desc(q_heads=hq, dtype=dt, scale=dim ** -0.5)
    ws = torch.empty(max(ctx.attn_workspace_bytes(attn, 3), ctx.scan_workspace_bytes(scan, 3, sum(lens)), 16), dtype=torch.uint8, device="cuda")
    r = _i32(reqs)

    def layer(x, n, cu):
        """x [n, 2 d] -> what every call put out."""
        tokens = x.shape[0]
        o = SimpleNamespace(x=x, y=torch.empty(tokens, d, dtype=dt, device="cuda"), s=torch.empty(tokens, d, dtype=dt, device="cuda"),
                            q=torch.empty(tokens, hq, dim, dtype=dt, device="cuda"), o=torch.empty(tokens, hq, dim, dtype=dt, device="cuda"))
        if cu is None:
            ctx.conv_step(0, conv, r, n, x, weight, bias, o.y)
        else:
            ctx.conv_prompt(0, conv, r, n, cu, tokens, None, x, weight, bias, o.y)
        o.p = o.y @ proj
        parts = (o.y, o.p, o.p[:, d:], o.p[:, d + ns:], x[:, d:], a, skip, None, o.s)
        if cu is None:
            ctx.scan_step(0, scan, r, n, *parts)
        else:
            ctx.scan_prompt(0, scan, r, n, cu, tokens, None, *parts, ws, ws.numel())
        o.qkv = o.s @ up
        q, k, v = o.qkv.split([hq * dim, hk * dim, hk * dim], 1)
        if cu is None:
            ctx.attn_rows_step(0, rows, r, n, None, q, k, v, wq, wk, freq, o.q)
            ctx.attn_window_decode(0, attn, window, sinks, r, n, o.q, o.o, None, ws, ws.numel())
        else:
            ctx.attn_rows_prompt(0, rows, r, n, cu, tokens, None, q, k, v, wq, wk, freq, o.q)
            ctx.attn_window_prompt(0, attn, window, sinks, r, n, cu, tokens, o.q, o.o, None, ws, ws.numel())
        return o

    cu = np.concatenate([[0], np.cumsum(lens)])
    xs = [(normal(sum(lens), 2 * d)).to(dt)] + [normal(3, 2 * d).to(dt) for _ in range(3)]
    side = torch.cuda.Stream()
    outs = []
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        o = layer(xs[0], 3, _i32(cu))
        outs.append(o)
        fixed = torch.zeros(3, 2 * d, dtype=dt, device="cuda")
        torch.zeros(3, d, dtype=dt, device="cuda") @ proj, torch.zeros(3, d, dtype=dt, device="cuda") @ up      # the library's matrix products warm up
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = layer(fixed, 3, None)
    for i in range(3):
        st[:] = 9
        ctx.step_host(W.make_ops(W.OP_EXTEND, reqs, [1, 1, 1]), 3, st, stream=side)
        assert (st == 0).all()
        with torch.cuda.stream(side):
            fixed.copy_(xs[1 + i])
            graph.replay()
            outs.append(SimpleNamespace(**{k: v.clone() for k, v in vars(captured).items()}))
    side.synchronize()
    assert ctx.stats()["error_count"] == 0
    for e in range(3):
        sl = slice(cu[e], cu[e + 1])
        line = lambda name: torch.cat([getattr(outs[0], name)[sl]] + [getattr(p, name)[e:e + 1] for p in outs[1:]])
        x, y, p, s, qkv, q, o = (line(n) for n in ("x", "y", "p", "s", "qkv", "q", "o"))
        want, bound, _ = _conv_exact(x[:, :d], torch.zeros(w - 1, d, device="cuda"), weight, bias, True)
        _near(y, want, bound, "convolution")
        _, _, want, bound = _scan_exact(torch.zeros(d, ns, device="cuda"), y, p[:, :d], p[:, None, d:d + ns], p[:, None, d + ns:], x[:, d:], a, skip, None,
                                        True)
        _near(s, want, bound, "scan")
        place = torch.arange(len(x), device="cuda")
        qq, kk, vv = (t.unflatten(1, (-1, dim)) for t in qkv.split([hq * dim, hk * dim, hk * dim], 1))
        _near(q, *_rotated(qq, wq, 1e-6, place, freq, False), "queries")
        k16 = _rotated(kk, wk, 1e-6, place, freq, False)[0].to(dt)
        want, _ = _exact(q, torch.stack([k16, vv]), dim ** -0.5, 0, window, sinks)
        # a key may be rounded the other way than here: eps/2 of a score's terms, next to the roundings of the weights
        assert float((o.double() - want).norm() / want.norm()) <= 4 * torch.finfo(dt).eps / 2, "attention"
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_long_lists_of_single_tokens(dtype):
    """Lists of more entries than a CTA looks after or plans by itself, with a slot out of range and repeated slots: the first of each is written."""
    import torch
    from paper_2605_22416_b200 import binding as B
    n, hk, hq, dim, window, sinks = 1600, 1, 2, 64, 9, 2
    rng = np.random.default_rng(4)
    held = [int(h) for h in rng.integers(1, 40, n)]
    c = Cache(held, hk, dim, 16, dtype, seed=1)
    reqs = rng.permutation(n)
    reqs[1100], reqs[7], reqs[1599] = 70000, reqs[5], reqs[300]
    bad = [7, 1100, 1599]
    q, k, v = (torch.randn(n, h, dim, device="cuda", generator=c.gen).to(c.dt) for h in (hq, hk, hk))
    freq = torch.rand(dim // 2, device="cuda", generator=c.gen)
    out = torch.full((n, hq, dim), 7.0, dtype=c.dt, device="cuda")
    c.ctx.attn_rows_step(c.layer, B.rows_desc(q_heads=hq, rotary_dim=dim, neighbours=False, eps=1e-6, dtype=c.dt), _i32(reqs), n, None, q, k, v,
                         None, None, freq, out)
    good = torch.tensor([e for e in range(n) if e not in bad], device="cuda")
    place = torch.tensor([held[r] - 1 if r < n else 0 for r in reqs], device="cuda")
    assert (out[bad] == 7).all() and c.ctx.stats()["error_count"] == 3
    want, bound = _rotated(q, None, 0, place, freq, False)
    _near(out[good], want[good], bound[good], "queries")
    want_k, bound_k = _rotated(k, None, 0, place, freq, False)
    c.ctx.clear_error()
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=dim ** -0.5)
    ws, size = c.workspace(desc, n)
    seen, lse = torch.full((n, hq, dim), 7.0, dtype=c.dt, device="cuda"), torch.empty(n, hq, device="cuda")
    c.ctx.attn_window_decode(c.layer, desc, window, sinks, _i32(reqs), n, out, seen, lse, ws, size)
    assert c.ctx.stats()["error_count"] == 1 and (seen[1100] == 7).all()
    for e in (0, 4, 5, 6, 300, 301, 777, 1099, 1101, 1598):
        r = int(reqs[e])
        kk, vv = _cached(c, r)
        assert torch.equal(kk[:-1], c.rows[r][0][:-1]) and torch.equal(vv[:-1], c.rows[r][1][:-1]) and torch.equal(vv[-1], v[e])
        _near(kk[-1:], want_k[e:e + 1], bound_k[e:e + 1], f"key of entry {e}")
        o, ll = _exact(out[e:e + 1], torch.stack([kk, vv]), dim ** -0.5, held[r] - 1, window, sinks)
        _check(seen[e:e + 1], lse[e:e + 1], o, ll, f"entry {e}")
    c.ctx.close()
