"""Convolution, selective scan, attention rows and window attention at sizes at which their kernels share out work otherwise than for the
small calls of test_conv_scan.py and test_rows_window.py: runs of many rows, copy rings that are filled several times over, several tokens or
entries for a CTA, lists of more entries than are looked up at a time, lanes of all states, tiles of whole prompts.  (How many rows, entries or
states go together follows from the number of SMs; the sizes are chosen for 148, and are right for any.)

References and tolerances are those of these two files: the formulas in 64 bits, bounds carried along entry by entry.
"""
from __future__ import annotations

import math

import numpy as np
import pytest

from test_attn_ops import Cache, _check, _i32
from test_conv_scan import _conv_exact, _fill, _inside, _model, _scan_desc, _scan_exact, _scan_inputs
from test_rows_window import _cached, _exact, _near, _rotated
from test_ssm_ops import _ctx, _rows, _states


def _offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)])


# ---------------------------------------------------------------- convolution
CONV = [
    # channels, width, lengths, rows of a run
    (2056, 4, [7000, 1, 40, 127, 128, 0, 129, 2, 9001, 131], 128),
    (1032, 3, [9000, 63, 10, 65, 2, 3600], 64),
    (2056, 2, [2500, 31, 20, 33, 1, 1300], 32),
    (520, 4, [3001, 15, 16, 17, 0, 1, 1700], 16),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(CONV)))
def test_conv_prompts_of_many_rows(dtype, case):
    """Runs of 16 to 128 rows: every place of the ring is filled again while others are worked on.  The third entry's slot is empty."""
    import torch
    from paper_2605_22416_b200 import binding as B
    d, w, lens, _ = CONV[case]
    dt, n = getattr(torch, dtype), len(lens)
    m = _model(d, 8, w, layers=1)
    reqs = [(7 * i + 3) % 13 for i in range(n)]
    live = [r for i, r in enumerate(reqs) if i != 2]
    ctx = _ctx(m, 13, live)
    gen = torch.Generator("cuda").manual_seed(case)
    st, cv = _fill(ctx, 0, live, m, gen, dt)
    at = {r: i for i, r in enumerate(live)}
    resume = [(i + 1) % 2 for i in range(n)]
    for i, r in enumerate(reqs):
        if i != 2 and not resume[i]:
            ctx.scatter_ssm(0, _i32([r]), 1, st[at[r]:at[r] + 1].contiguous(), torch.full((1, m.ssm_conv_elems), math.nan, device="cuda"))
    cu, tot = _offsets(lens), sum(lens)
    x, xs = _rows((tot, d), dt, gen, 1.0, pad=24)
    weight, bias = torch.randn(d, w, device="cuda", generator=gen), torch.randn(d, device="cuda", generator=gen)
    out = torch.full((tot + 2, d + 8), 7.0, dtype=dt, device="cuda")
    desc = B.conv_desc(channels=d, width=w, silu=True, dtype=dt, x_stride_bytes=xs, out_stride_bytes=(d + 8) * 2)
    ctx.conv_prompt(0, desc, _i32(reqs), n, _i32(cu), tot, _i32(resume), x, weight, bias, out)
    st2, cv2 = _states(ctx, 0, live, m)
    assert torch.equal(st2, st) and ctx.stats()["error_count"] == 1
    for i, r in enumerate(reqs):
        sl = slice(cu[i], cu[i + 1])
        if i == 2:
            assert (out[sl] == 7).all()
            continue
        y, bound, new = _conv_exact(x[sl], cv[at[r]].view(w - 1, d) * resume[i], weight, bias, True)
        _inside(out[sl, :d], y, bound, dt, f"rows of {i}")
        assert torch.equal(cv2[at[r]].view(w - 1, d).double(), new), i
    assert (out[:, d:] == 7).all() and (out[tot:] == 7).all()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n", [501, 954])
def test_conv_steps_of_many_requests(dtype, n):
    """Two and four entries for a CTA, repeated, empty and impossible slots among them."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt, d, w = getattr(torch, dtype), 2056, 4
    m = _model(d, 8, w, layers=1)
    ctx = _ctx(m, n + 1, range(n))
    gen = torch.Generator("cuda").manual_seed(n)
    st, cv = _fill(ctx, 0, range(n), m, gen, dt)
    reqs = np.random.default_rng(n).permutation(n).astype(np.int64)
    bad = [2, n // 3, n // 2, n - 1]
    reqs[bad] = [reqs[1], n, reqs[0], 0xFFFFFFFF]
    good = [e for e in range(n) if e not in bad]
    x = torch.randn(n, d, device="cuda", generator=gen).to(dt)
    weight, bias = torch.randn(d, w, device="cuda", generator=gen), torch.randn(d, device="cuda", generator=gen)
    out = torch.full((n, d), 7.0, dtype=dt, device="cuda")
    ctx.conv_step(0, B.conv_desc(channels=d, width=w, silu=True, dtype=dt), _i32(reqs), n, x, weight, bias, out)
    slot = torch.tensor(reqs[good], device="cuda")
    old = cv.view(n, w - 1, d)[slot]
    k = len(good)
    y, bound, _ = _conv_exact(x[good].reshape(1, k * d), old.transpose(0, 1).reshape(w - 1, k * d), weight.repeat(k, 1), bias.repeat(k), True)
    _inside(out[good].reshape(1, -1), y, bound, dt, "rows")
    want = cv.view(n, w - 1, d).clone()
    want[slot] = torch.cat([old[:, 1:], x[good][:, None].float()], 1)
    st2, cv2 = _states(ctx, 0, range(n), m)
    assert torch.equal(st2, st) and torch.equal(cv2.view(n, w - 1, d), want)
    assert (out[bad] == 7).all() and ctx.stats()["error_count"] == 4
    ctx.close()


# ---------------------------------------------------------------- scan
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,d,g,states", [(600, 2048, 1, 16), (700, 4096, 2, 8), (600, 1048, 1, 32), (300, 1040, 1, 64), (5000, 256, 32, 8)])
def test_scan_steps_of_many_requests(dtype, n, d, g, states):
    """Ten to five hundred entries for a CTA: the ring goes round, decays stay from entry to entry and change with the tile, and the last list is longer
    than what is looked up at a time.  Repeated, empty and impossible slots among the entries."""
    import torch
    dt = getattr(torch, dtype)
    m = _model(d, states, 2, layers=1)
    ctx = _ctx(m, n + 1, range(n))
    gen = torch.Generator("cuda").manual_seed(n + d)
    st, cv = _fill(ctx, 0, range(n), m, gen, dt)
    reqs = np.random.default_rng(n).permutation(n).astype(np.int64)
    bad = [4, n // 3, n // 2, n - 2]
    reqs[bad] = [reqs[3], n, reqs[1], 0xFFFFFFFF]
    good = [e for e in range(n) if e not in bad]
    i = _scan_inputs(d, g, states, n, dt, gen)
    out = torch.full((n, d), 7.0, dtype=dt, device="cuda")
    ctx.scan_step(0, _scan_desc(i, d, g, states, dt), _i32(reqs), n, i.u, i.delta, i.b, i.c, i.z, i.a, i.skip, i.bias, out)
    st2, cv2 = _states(ctx, 0, range(n), m)
    named = torch.zeros(n, dtype=torch.bool, device="cuda")
    for part in np.array_split(np.asarray(good), 8):       # the entries' channels side by side: one request of that many channels and groups
        k, slot, part = len(part), torch.tensor(reqs[part], device="cuda"), torch.tensor(part, device="cuda")
        named[slot] = True
        line = lambda x: x[part].reshape(1, -1)
        h, err, y, bound = _scan_exact(st[slot].view(k * d, states), line(i.u), line(i.delta), i.b[part].reshape(1, k * g, states),
                                       i.c[part].reshape(1, k * g, states), line(i.z), i.a.repeat(k, 1), i.skip.repeat(k), i.bias.repeat(k), True)
        _inside(st2[slot].view(k * d, states), h, err, None, "states")
        _inside(line(out), y, bound, dt, "rows")
    assert torch.equal(st2[~named], st[~named]) and int(named.sum()) == n - 4
    assert torch.equal(cv2, cv) and (out[bad] == 7).all() and ctx.stats()["error_count"] == 4
    ctx.close()


SCAN = [
    # requests, channels, groups, states, longest: lanes of all states (32 and 64: of 16)
    (100, 200, 5, 8, 90),
    (100, 200, 5, 16, 90),
    (150, 120, 3, 32, 60),
    (150, 120, 3, 64, 60),
    # the same, prompts cut into runs
    (20, 256, 1, 16, 1000),
    (20, 128, 1, 32, 1000),
    (20, 64, 1, 64, 1000),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(SCAN)))
def test_scan_prompts_of_many_channels(dtype, case):
    import torch
    n, d, g, states, most = SCAN[case]
    dt = getattr(torch, dtype)
    m = _model(d, states, 2, layers=1)
    ctx = _ctx(m, n + 1, range(n))
    gen = torch.Generator("cuda").manual_seed(case)
    st, cv = _fill(ctx, 0, range(n), m, gen, dt)
    rng = np.random.default_rng(case)
    reqs = rng.permutation(n).astype(np.int64)
    lens = rng.integers(0, most // 2, n) + (most // 4 if case > 3 else 0)
    lens[[1, 5, 7, n - 1]] = most, 1, 0, most - 1
    bad = [3, 10]
    reqs[bad] = n, reqs[2]
    cu, tot = _offsets(lens), int(lens.sum())
    resume = rng.integers(0, 2, n)
    i = _scan_inputs(d, g, states, tot, dt, gen)
    out = torch.full((tot + 1, d), 7.0, dtype=dt, device="cuda")
    desc = _scan_desc(i, d, g, states, dt)
    size = ctx.scan_workspace_bytes(desc, n, tot)
    ws = torch.full((max(16, size),), 0xFF, dtype=torch.uint8, device="cuda")
    ctx.scan_prompt(0, desc, _i32(reqs), n, _i32(cu), tot, _i32(resume), i.u, i.delta, i.b, i.c, i.z, i.a, i.skip, i.bias, out, ws, size)
    st2, cv2 = _states(ctx, 0, range(n), m)
    for e in sorted({0, 1, 2, 3, 5, 7, 10, 11, n // 2, n - 2, n - 1}):
        r, sl = int(reqs[e]), slice(cu[e], cu[e + 1])
        if e in bad:
            assert (out[sl] == 7).all()
            continue
        h, err, y, bound = _scan_exact(st[r].view(d, states) * int(resume[e]), i.u[sl], i.delta[sl], i.b[sl].unflatten(1, (g, states)),
                                       i.c[sl].unflatten(1, (g, states)), i.z[sl], i.a, i.skip, i.bias, True)
        _inside(st2[r].view(d, states), h, err, None, f"state {e}")
        _inside(out[sl], y, bound, dt, f"rows of {e}")
    assert torch.isfinite(out).all() and (out[tot:] == 7).all() and torch.equal(cv2, cv) and ctx.stats()["error_count"] == 2
    ctx.close()


# ---------------------------------------------------------------- rows
ROWS = [
    # new, kv_heads, group, dim, page, rotary, neighbours, norm: two tokens a CTA, then four
    ([700, 1, 40, 2, 3, 501, 0, 298], 8, 8, 128, 16, 128, False, True),
    ([1501, 1, 40, 2, 3, 997, 0, 514], 8, 8, 128, 32, 64, True, True),
    ([5, 2400, 30, 1, 6, 239], 4, 12, 64, 16, 64, False, True),
    ([1301, 7, 40, 2, 1250], 2, 20, 64, 8, 16, True, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(ROWS)))
def test_rows_of_long_prompts(dtype, case):
    """Warps with a token each, or two, and so many heads that the ring goes round.  The third entry's slot is empty."""
    import torch
    from paper_2605_22416_b200 import binding as B
    new, hk, group, dim, page, rotary, neighbours, norm = ROWS[case]
    n, hq, tot, cu = len(new), hk * group, sum(new), _offsets(new)
    held = [0 if i == 2 else a + 13 * i for i, a in enumerate(new)]
    held = [h + 1 if i != 2 and h == 0 else h for i, h in enumerate(held)]
    c = Cache(held, hk, dim, page, dtype, seed=case)
    width = (hq + 2 * hk) * dim
    qkv = torch.randn(tot, width + 16, device="cuda", generator=c.gen).to(c.dt)
    q, k, v = (x.unflatten(1, (-1, dim)) for x in qkv[:, :width].split([hq * dim, hk * dim, hk * dim], 1))
    wq, wk = ((1 + 0.3 * torch.randn(dim, device="cuda", generator=c.gen)) if norm else None for _ in range(2))
    freq = (10000.0 ** (-torch.arange(rotary // 2, device="cuda") / (rotary // 2))).float()
    out = torch.full((tot + 1, hq, dim), 7.0, dtype=c.dt, device="cuda")
    stride = (width + 16) * 2
    desc = B.rows_desc(q_heads=hq, rotary_dim=rotary, neighbours=neighbours, eps=1e-5, dtype=c.dt, q_stride_bytes=stride, k_stride_bytes=stride,
                       v_stride_bytes=stride)
    c.ctx.attn_rows_prompt(c.layer, desc, _i32(range(n)), n, _i32(cu), tot, None, q, k, v, wq, wk, freq, out)
    for r in range(n):
        sl = slice(cu[r], cu[r + 1])
        if r == 2:
            assert (out[sl] == 7).all()
            continue
        kk, vv = _cached(c, r)
        old = held[r] - new[r]
        assert torch.equal(kk[:old], c.rows[r][0][:old]) and torch.equal(vv[:old], c.rows[r][1][:old])
        if new[r]:
            place = torch.arange(old, held[r], device="cuda")
            _near(out[sl], *_rotated(q[sl], wq, 1e-5, place, freq, neighbours), f"queries of {r}")
            _near(kk[old:], *_rotated(k[sl], wk, 1e-5, place, freq, neighbours), f"keys of {r}")
            assert torch.equal(vv[old:], v[sl])
    assert (out[tot:] == 7).all() and c.ctx.stats()["error_count"] == 1
    c.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,hk,group,dim,neighbours", [(1201, 8, 8, 128, False), (3001, 4, 12, 64, True)])
def test_rows_of_many_single_tokens(dtype, n, hk, group, dim, neighbours):
    """Two and four entries for a CTA, many heads; repeated, empty and impossible slots."""
    import torch
    from paper_2605_22416_b200 import binding as B
    rng = np.random.default_rng(n)
    few = [int(h) for h in rng.integers(1, 20, 64)]
    c = Cache([few[i % 64] for i in range(n)], hk, dim, 16, dtype, seed=1)
    hq = hk * group
    reqs = rng.permutation(n).astype(np.int64)
    bad = [6, n // 3, n // 2, n - 1]
    reqs[bad] = reqs[5], n + 1, reqs[0], 70000
    good = torch.tensor([e for e in range(n) if e not in bad], device="cuda")
    q, k, v = (torch.randn(n, h, dim, device="cuda", generator=c.gen).to(c.dt) for h in (hq, hk, hk))
    wq, wk = (1 + 0.3 * torch.randn(dim, device="cuda", generator=c.gen) for _ in range(2))
    freq = torch.rand(dim // 2, device="cuda", generator=c.gen)
    out = torch.full((n, hq, dim), 7.0, dtype=c.dt, device="cuda")
    desc = B.rows_desc(q_heads=hq, rotary_dim=dim, neighbours=neighbours, eps=1e-6, dtype=c.dt)
    c.ctx.attn_rows_step(c.layer, desc, _i32(reqs), n, None, q, k, v, wq, wk, freq, out)
    place = torch.tensor([c.held[r] - 1 if r < n else 0 for r in reqs], device="cuda")
    want, bound = _rotated(q[good], wq, 1e-6, place[good], freq, neighbours)
    _near(out[good], want, bound, "queries")
    assert (out[bad] == 7).all() and c.ctx.stats()["error_count"] == 4
    want, bound = _rotated(k, wk, 1e-6, place, freq, neighbours)
    for e in (0, 1, 2, 3, 4, 5, 7, n // 3 - 1, n // 3 + 1, 777, n - 5, n - 4, n - 3, n - 2):
        kk, vv = _cached(c, int(reqs[e]))
        old = c.rows[int(reqs[e])]
        _near(kk[-1:], want[e:e + 1], bound[e:e + 1], f"key of {e}")
        assert torch.equal(vv[-1], v[e]) and torch.equal(kk[:-1], old[0][:-1]) and torch.equal(vv[:-1], old[1][:-1])
    c.ctx.close()


# ---------------------------------------------------------------- window
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,hk,group,dim,page", [(12, 8, 4, 128, 16), (40, 2, 8, 128, 32), (9, 16, 3, 64, 8), (10, 4, 8, 64, 24)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (60, 5), (257, 129), (1024, 4), (1 << 20, 1)])
def test_window_prompts_of_whole_tiles(dtype, n, hk, group, dim, page, window, sinks):
    """Enough tiles for all SMs, so that none is split: up to 32 requests handed out without a list, more with one.  What no row of a request sees
    is NaN in the cache; the second request's slot is empty."""
    import torch
    from paper_2605_22416_b200 import binding as B
    rng = np.random.default_rng(n)
    new = [int(x) for x in rng.integers(150, 400, n)] if n < 40 else [int(x) for x in rng.integers(70, 130, n)]
    new[0], new[3], new[4] = 700, 1, 0
    held = [a + int(p) for a, p in zip(new, rng.integers(0, 1500, n))]
    held[1], held[5] = 0, new[5]
    held[4] = max(1, held[4])
    c = Cache(held, hk, dim, page, dtype, seed=n)
    hq, scale, tot, cu = hk * group, dim ** -0.5, sum(new), _offsets(new)
    q, qs = c.queries(tot, hq, pad=8)
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=scale, q_stride_bytes=qs)
    out, lse = torch.full((tot + 1, hq, dim), 7.0, dtype=c.dt, device="cuda"), torch.full((tot + 1, hq), 7.0, device="cuda")
    ws, size = c.workspace(desc, n)
    live = [r for r in range(n) if held[r] and new[r]]
    want = {r: _exact(q[cu[r]:cu[r + 1]], c.rows[r], scale, held[r] - new[r], window, sinks) for r in live}
    for r in live:
        j, first = torch.arange(held[r], device="cuda"), held[r] - new[r]
        hidden = (j < first + 1 - min(window, first + 1)) & (j >= sinks)
        if hidden.any():
            kv = c.rows[r].clone()
            kv[:, hidden] = math.nan
            c.ctx.scatter_kv(c.layer, _i32([r]), None, 1, kv[0].contiguous(), kv[1].contiguous())
    c.ctx.attn_window_prompt(c.layer, desc, window, sinks, _i32(range(n)), n, _i32(cu), tot, q, out, lse, ws, size)
    for r in live:
        sl = slice(cu[r], cu[r + 1])
        _check(out[sl], lse[sl], *want[r], f"request {r}")
    assert (out[cu[1]:cu[2]] == 7).all() and (lse[cu[1]:cu[2]] == 7).all() and (out[tot:] == 7).all() and (lse[tot:] == 7).all()
    assert c.ctx.stats()["error_count"] == 1
    c.ctx.close()


@pytest.mark.gpu
def test_rows_of_offsets_that_swing():
    """Offsets that run over all of 2^28 rows and back, again and again: skipped items, whose runs together pass 2^32.  The one good entry behind
    them is served."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dim, n, tot = 64, 129, (1 << 28) + 64
    c = Cache([40] + [1] * (n - 1), 1, dim, 16, "bfloat16")
    freq = torch.rand(dim // 2, device="cuda", generator=c.gen)
    x, out = (torch.empty(tot, 1, dim, dtype=c.dt, device="cuda") for _ in range(2))
    x[:64] = torch.randn(64, 1, dim, device="cuda", generator=c.gen).to(c.dt)
    out[:64] = 7.0
    cu = [0, tot] * (n // 2) + [0, 40]
    reqs = list(range(1, n)) + [0]
    desc = B.rows_desc(q_heads=1, rotary_dim=dim, neighbours=False, eps=1e-6, dtype=c.dt)
    c.ctx.attn_rows_prompt(c.layer, desc, _i32(reqs), n, _i32(cu), tot, None, x, x, x, None, None, freq, out)
    assert c.ctx.stats()["error_count"] == n - 1
    want, bound = _rotated(x[:40], None, 0, torch.arange(40, device="cuda"), freq, False)
    _near(out[:40], want, bound, "queries")
    assert (out[40:64] == 7).all() and torch.equal(_cached(c, 0)[1], x[:40])
    c.ctx.close()
    del x, out
    torch.cuda.empty_cache()
