"""Short convolution and selective scan on the SSM blocks (avmp_conv_*, avmp_scan_*) against their formulas in 64 bits, token by token.

Tolerances are bounds carried along with the 64-bit values, entry by entry.
Convolution: at most 5 roundings (2^-24 each) of sums of |w x| and |b|, the gate's exponential and reciprocal (2^-21 together), one
rounding to 16 bits.  The window holds 16-bit numbers: equal.
Scan, per token: the step is off by r = (|delta + bias| + 16) 2^-24 (rounding of its argument, expf and log1pf of a few 2^-24), a decay by
c = 2^-22 + |step A| (r + 2^-22) (the exponential, and its argument's error), what is added by r + 2^-22, the sum by 2^-24.  An output
is a sum of `states` products of that (states 2^-24 more), gated (2^-21) and rounded once.
fp16 results below its normal range are off by 2^-25 at most.
"""
from __future__ import annotations

import math

import numpy as np
import pytest

from test_ssm_ops import _ctx, _i32, _rows, _states
from types import SimpleNamespace

ULP = 2.0 ** -24


def _model(channels, states, width, layers=2):
    return SimpleNamespace(n_attn_layers=1, n_ssm_layers=layers, page_tokens=16, kv_heads=1, head_dim=64, kv_elem_bytes=2,
                           ssm_state_elems=channels * states, ssm_conv_elems=channels * (width - 1), ssm_elem_bytes=4)


def _fill(ctx, layer, reqs, m, gen, dt):
    """Blocks with random states and windows of 16-bit numbers."""
    import torch
    st = torch.randn(len(reqs), m.ssm_state_elems, device="cuda", generator=gen)
    cv = torch.randn(len(reqs), m.ssm_conv_elems, device="cuda", generator=gen).to(dt).float()
    ctx.scatter_ssm(layer, _i32(reqs), len(reqs), st, cv)
    return st, cv


def _inside(got, want, bound, dt, what):
    """|got - want| <= bound, then one rounding to dt (None: none)."""
    import torch
    if got.numel() == 0:
        return
    assert torch.isfinite(got).all(), what
    off = (got.double() - want).abs()
    allowed = bound if dt is None else bound + (want.abs() + bound) * (torch.finfo(dt).eps / 2) + 2.0 ** -25
    worst = float((off - allowed).max())
    assert worst <= 0, f"{what}: {worst:.3g} over the bound, off by {float(off.max()):.3g}"


def _conv_exact(x, window, weight, bias, act):
    """x [L, d], window [w - 1, d] -> out, bound, window."""
    import torch
    w = weight.shape[1]
    line = torch.cat([window.double(), x.double()])
    taps = [line[j: j + x.shape[0]] * weight[:, j].double() for j in range(w)]
    b = 0 if bias is None else bias.double()
    y, size = sum(taps) + b, sum(t.abs() for t in taps) + (0 if bias is None else b.abs())
    bound = 5 * ULP * size
    if act:
        # the gate's slope is at most 1.1
        y, bound = y * torch.sigmoid(y), 1.1 * bound + 2.0 ** -21 * y.abs()
    return y, bound, line[x.shape[0]:]


def _scan_exact(h, u, delta, b, c, z, a, skip, bias, softplus):
    """One request: h [d, n]; u, delta, z [L, d]; b, c [L, g, n] -> state, its bound, out, its bound."""
    import torch
    d, n = h.shape
    rep = d // b.shape[1]
    h, a = h.double(), a.double()
    err = torch.zeros_like(h)
    outs, bounds = [], []
    for t in range(u.shape[0]):
        v = delta[t].double() + (0 if bias is None else bias.double())
        step = torch.logaddexp(v, torch.zeros_like(v)) if softplus else v
        r = ((v.abs() + 16) * ULP)[:, None]
        x = step[:, None] * a
        decay = x.exp()
        add = (step * u[t].double())[:, None] * b[t].double().repeat_interleave(rep, 0)
        err = decay * (err + h.abs() * (2.0 ** -22 + x.abs() * (r + 2.0 ** -22))) + add.abs() * (r + 2.0 ** -22)
        h = decay * h + add
        err = err + h.abs() * ULP
        cc = c[t].double().repeat_interleave(rep, 0)
        y, e = (h * cc).sum(-1), (cc.abs() * (err + h.abs() * n * ULP)).sum(-1)
        if skip is not None:
            p = skip.double() * u[t].double()
            y, e = y + p, e + (p.abs() + y.abs()) * 2 * ULP
        if z is not None:
            gate = z[t].double() * torch.sigmoid(z[t].double())
            y, e = y * gate, (e + y.abs() * 2.0 ** -21) * gate.abs()
        outs.append(y)
        bounds.append(e)
    empty = torch.zeros(0, d, dtype=torch.float64, device=h.device)
    return h, err, torch.stack(outs) if outs else empty, torch.stack(bounds) if bounds else empty


CONV = [
    # channels, width, lengths, resume, bias, silu
    (8, 2, [1], [0], False, False),
    (16, 4, [0, 1, 2, 3, 4, 9], [0, 1, 0, 1, 0, 1], True, True),
    (1032, 4, [65, 0, 200], [1, 1, 0], True, True),
    (72, 3, [1, 1, 130, 2], [1, 0, 1, 1], False, True),
    (2048, 4, [700, 1, 64, 63], [1, 0, 1, 0], True, False),
    (264, 2, [5, 0, 33], [0, 1, 1], True, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(CONV)))
def test_conv_prompts(dtype, case):
    import torch
    from paper_2605_22416_b200 import binding as B
    d, w, lens, resume, with_bias, act = CONV[case]
    dt = getattr(torch, dtype)
    m = _model(d, 8, w)
    reqs = [(5 * i + 3) % 13 for i in range(len(lens))]
    ctx = _ctx(m, 13, reqs + [12])
    gen = torch.Generator("cuda").manual_seed(case)
    st, cv = _fill(ctx, 1, reqs, m, gen, dt)
    other = _fill(ctx, 0, reqs, m, gen, dt)
    bystander = _fill(ctx, 1, [12], m, gen, dt)
    for i in range(len(lens)):
        if not resume[i]:        # what a fresh block holds is not read
            ctx.scatter_ssm(1, _i32([reqs[i]]), 1, st[i:i + 1].contiguous(), torch.full((1, m.ssm_conv_elems), math.nan, device="cuda"))
    tot = sum(lens)
    x, xs = _rows((tot, d), dt, gen, 1.0, pad=8 * case)
    weight = torch.randn(d, w, device="cuda", generator=gen)
    bias = torch.randn(d, device="cuda", generator=gen) if with_bias else None
    out = torch.full((tot + 2, d + 8), 7.0, dtype=dt, device="cuda")
    desc = B.conv_desc(channels=d, width=w, silu=act, dtype=dt, x_stride_bytes=xs, out_stride_bytes=(d + 8) * 2)
    cu = np.concatenate([[0], np.cumsum(lens)])
    ctx.conv_prompt(1, desc, _i32(reqs), len(lens), _i32(cu), tot, _i32(resume), x, weight, bias, out)
    st2, cv2 = _states(ctx, 1, reqs, m)
    assert torch.equal(st2, st)
    for i, n in enumerate(lens):
        old = cv[i].view(w - 1, d) * resume[i]
        y, bound, new = _conv_exact(x[cu[i]:cu[i + 1]], old, weight, bias, act)
        _inside(out[cu[i]:cu[i + 1], :d], y, bound, dt, f"rows of {i}")
        assert torch.equal(cv2[i].view(w - 1, d).double(), new), i
    assert (out[:, d:] == 7).all() and (out[tot:] == 7).all()
    for layer, rs, was in ((0, reqs, other), (1, [12], bystander)):
        assert all(torch.equal(p, q) for p, q in zip(_states(ctx, layer, rs, m), was))
    assert ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,d,w", [(1, 8, 4), (5, 1032, 3), (37, 520, 4), (300, 2048, 2)])
def test_conv_steps(dtype, n, d, w):
    """Three tokens one after the other; a repeated slot, an empty one and one out of range are skipped and counted."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = getattr(torch, dtype)
    m = _model(d, 8, w, layers=1)
    order = np.random.default_rng(n).permutation(n)
    ctx = _ctx(m, n + 3, order)
    gen = torch.Generator("cuda").manual_seed(n)
    st, cv = _fill(ctx, 0, order, m, gen, dt)
    reqs = list(order) + ([order[0], n + 1, 0xFFFFFFFF] if n > 4 else [])
    k = min(len(reqs), n + 3)
    weight, bias = torch.randn(d, w, device="cuda", generator=gen), torch.randn(d, device="cuda", generator=gen)
    desc = B.conv_desc(channels=d, width=w, silu=True, dtype=dt)
    window = cv.view(n, w - 1, d)
    for step in range(3):
        x = torch.randn(k, d, device="cuda", generator=gen).to(dt)
        out = torch.full((k, d), 7.0, dtype=dt, device="cuda")
        ctx.conv_step(0, desc, _i32(reqs), k, x, weight, bias, out)
        line = torch.cat([window, x[:n, None].float()], 1)
        y, bound, _ = _conv_exact(x[:n].reshape(1, n * d), window.transpose(0, 1).reshape(w - 1, n * d), weight.repeat(n, 1), bias.repeat(n), True)
        _inside(out[:n].reshape(1, -1), y, bound, dt, f"token {step}")
        window = line[:, 1:]
        assert (out[n:] == 7).all() and ctx.stats()["error_count"] == (k - n) * (step + 1)
    st2, cv2 = _states(ctx, 0, order, m)
    assert torch.equal(st2, st) and torch.equal(cv2.view(n, w - 1, d), window)
    ctx.close()


def _scan_inputs(d, g, n, tot, dt, gen, mixed=0.0):
    """Rows inside wider buffers; the gate and B, C as slices of one projection each."""
    import torch
    normal = lambda *shape, scale=1.0: torch.randn(*shape, device="cuda", generator=gen) * scale
    i = SimpleNamespace()
    i.u, i.us = _rows((tot, d), dt, gen, 1.0, pad=8)
    i.delta, i.ds = _rows((tot, d), dt, gen, 1.0, pad=24)
    xz = normal(tot, 2 * d).to(dt)
    i.z, i.zs = xz[:, d:], 4 * d
    bc = normal(tot, 16 + 2 * g * n).to(dt)
    i.b, i.c, i.bs = bc[:, 16: 16 + g * n], bc[:, 16 + g * n:], (16 + 2 * g * n) * 2
    i.a = -torch.exp(normal(d, n) * 0.7)
    i.skip, i.bias = normal(d), normal(d) - 2.0
    return i


def _scan_desc(i, d, g, n, dt, softplus=True, **kw):
    from paper_2605_22416_b200 import binding as B
    return B.scan_desc(channels=d, groups=g, states=n, softplus=softplus, dtype=dt, u_stride_bytes=i.us, delta_stride_bytes=i.ds,
                       z_stride_bytes=i.zs, b_stride_bytes=i.bs, c_stride_bytes=i.bs, **kw)


SCAN = [
    # channels, groups, states, lengths, resume, softplus, gate, skip, bias
    (8, 1, 16, [1], [0], True, True, True, True),
    (40, 1, 16, [0, 1, 31, 32, 33, 100], [0, 1, 0, 1, 1, 0], True, True, True, True),
    (48, 2, 8, [65, 2, 0, 128], [1, 1, 1, 0], False, True, False, False),
    (104, 1, 32, [130, 7], [0, 1], True, False, True, True),
    (32, 4, 64, [97, 1, 40], [1, 0, 1], True, True, True, False),
    (2056, 1, 16, [300, 64, 12], [1, 1, 0], True, True, False, True),
    (240, 3, 16, [40] * 40, [1, 0] * 20, True, True, True, True),
    # few channels, long: cut into runs
    (64, 1, 16, [3000, 5, 0, 700], [1, 1, 1, 0], True, True, True, True),
    (24, 1, 64, [2500], [1], True, False, False, True),
    (16, 2, 8, [4097, 1], [0, 0], True, True, True, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(SCAN)))
def test_scan_prompts(dtype, case):
    import torch
    d, g, n, lens, resume, softplus, gate, skip, bias = SCAN[case]
    dt = getattr(torch, dtype)
    m = _model(d, n, 2)
    slots = max(13, len(lens) + 1)
    reqs = [(5 * i + 3) % 13 for i in range(len(lens))] if len(lens) < 13 else list(np.random.default_rng(1).permutation(len(lens)))
    stranger = next(r for r in range(slots) if r not in reqs)
    ctx = _ctx(m, slots, reqs + [stranger])
    gen = torch.Generator("cuda").manual_seed(case)
    st, cv = _fill(ctx, 1, reqs, m, gen, dt)
    other = _fill(ctx, 0, reqs, m, gen, dt)
    bystander = _fill(ctx, 1, [stranger], m, gen, dt)
    for i in range(len(lens)):
        if not resume[i]:
            ctx.scatter_ssm(1, _i32([reqs[i]]), 1, torch.full((1, m.ssm_state_elems), math.nan, device="cuda"), cv[i:i + 1].contiguous())
    tot = sum(lens)
    i = _scan_inputs(d, g, n, tot, dt, gen)
    if not softplus:
        i.delta = torch.nn.functional.softplus(i.delta.float() - 2).to(dt)
        i.ds = 0
    z, sk, bi = i.z if gate else None, i.skip if skip else None, i.bias if bias else None
    out = torch.full((tot + 2, d + 8), 7.0, dtype=dt, device="cuda")
    desc = _scan_desc(i, d, g, n, dt, softplus, out_stride_bytes=(d + 8) * 2)
    size = ctx.scan_workspace_bytes(desc, len(lens), tot)
    assert size > 0 or case < 7
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if size else None
    cu = np.concatenate([[0], np.cumsum(lens)])
    ctx.scan_prompt(1, desc, _i32(reqs), len(lens), _i32(cu), tot, _i32(resume), i.u, i.delta, i.b, i.c, z, i.a, sk, bi, out, ws, size)
    st2, cv2 = _states(ctx, 1, reqs, m)
    assert torch.equal(cv2, cv)
    for e in range(len(lens)):
        r = slice(cu[e], cu[e + 1])
        first = st[e].view(d, n) * resume[e]
        h, err, y, bound = _scan_exact(first, i.u[r], i.delta[r], i.b[r].unflatten(1, (g, n)), i.c[r].unflatten(1, (g, n)),
                                       None if z is None else z[r], i.a, sk, bi, softplus)
        _inside(st2[e].view(d, n), h, err, None, f"state {e}")
        _inside(out[r, :d], y, bound, dt, f"rows of {e}")
    assert (out[:, d:] == 7).all() and (out[tot:] == 7).all()
    for layer, rs, was in ((0, reqs, other), (1, [stranger], bystander)):
        assert all(torch.equal(p, q) for p, q in zip(_states(ctx, layer, rs, m), was))
    assert ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,d,g,states", [(1, 8, 1, 8), (6, 72, 1, 16), (33, 96, 3, 32), (130, 1000, 1, 16), (9, 48, 2, 64)])
def test_scan_steps(dtype, n, d, g, states):
    import torch
    dt = getattr(torch, dtype)
    m = _model(d, states, 2, layers=1)
    order = np.random.default_rng(n).permutation(n)
    ctx = _ctx(m, n + 3, order)
    gen = torch.Generator("cuda").manual_seed(n)
    st, cv = _fill(ctx, 0, order, m, gen, dt)
    reqs = list(order) + ([order[0], n + 1, 0xFFFFFFFF] if n > 4 else [])
    k = len(reqs)
    i = _scan_inputs(d, g, states, k, dt, gen)
    out = torch.full((k, d), 7.0, dtype=dt, device="cuda")
    ctx.scan_step(0, _scan_desc(i, d, g, states, dt), _i32(reqs), k, i.u, i.delta, i.b, i.c, i.z, i.a, i.skip, i.bias, out)
    st2, cv2 = _states(ctx, 0, order, m)
    for e in range(n):
        r = slice(e, e + 1)
        h, err, y, bound = _scan_exact(st[e].view(d, states), i.u[r], i.delta[r], i.b[r].unflatten(1, (g, states)), i.c[r].unflatten(1, (g, states)),
                                       i.z[r], i.a, i.skip, i.bias, True)
        _inside(st2[e].view(d, states), h, err, None, f"state {e}")
        _inside(out[r], y, bound, dt, f"row {e}")
    assert torch.equal(cv2, cv) and (out[n:] == 7).all() and ctx.stats()["error_count"] == k - n
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("op", ["conv", "scan", "scan_runs"])
def test_bad_items_of_prompts_are_skipped(op):
    """A slot that is not live, one out of range, one named before, offsets that decrease or pass the rows; the others' results stand."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = torch.bfloat16
    d, n, w = (8, 16, 4) if op == "scan_runs" else (64, 16, 4)
    m = _model(d, n, w, layers=1)
    ctx = _ctx(m, 12, [1, 2, 3, 4, 5])
    gen = torch.Generator("cuda").manual_seed(3)
    st, cv = _fill(ctx, 0, [1, 2, 3, 4, 5], m, gen, dt)
    long = 9000 if op == "scan_runs" else 40
    reqs = [1, 9, 2, 1, 77, 3, 4, 5]
    cu = [0, 20, 40, 30, 50, 60, 60 + long, 10 ** 6, 60]       # 2: decreasing, 4: past the rows, 5: decreasing from there
    tot = 60 + long
    i = _scan_inputs(d, 1, n, tot, dt, gen)
    out = torch.full((tot, d), 7.0, dtype=dt, device="cuda")
    if op == "conv":
        weight = torch.randn(d, w, device="cuda", generator=gen)
        desc = B.conv_desc(channels=d, width=w, silu=True, dtype=dt, x_stride_bytes=i.us)
        call = lambda rs, c, o: ctx.conv_prompt(0, desc, _i32(rs), len(rs), _i32(c), tot, _i32([1] * len(rs)), i.u, weight, None, o)
    else:
        desc = _scan_desc(i, d, 1, n, dt)
        size = ctx.scan_workspace_bytes(desc, len(reqs), tot)
        assert size > 0 or op == "scan"
        ws = torch.full((max(16, size),), 0xFF, dtype=torch.uint8, device="cuda")
        call = lambda rs, c, o: ctx.scan_prompt(0, desc, _i32(rs), len(rs), _i32(c), tot, _i32([1] * len(rs)), i.u, i.delta, i.b, i.c, i.z,
                                                i.a, i.skip, i.bias, o, ws, size)
    call(reqs, cu, out)
    assert ctx.stats()["error_count"] == 6 and ctx.stats()["error_code"] == 2
    got = _states(ctx, 0, [1, 2, 3, 4, 5], m)
    # requests 1 and 3 had rows of their own: the same as in calls without the others, from the same blocks
    ctx.scatter_ssm(0, _i32([1, 2, 3, 4, 5]), 5, st, cv)
    want = torch.full((tot, d), 7.0, dtype=dt, device="cuda")
    if op == "scan_runs":      # another number of entries may cut prompts otherwise: compare with the recurrence
        for e, c0, c1, r in ((0, 0, 20, 0), (2, 60, tot, 2)):
            h, err, y, bound = _scan_exact(st[e].view(d, n), i.u[c0:c1], i.delta[c0:c1], i.b[c0:c1, None], i.c[c0:c1, None], i.z[c0:c1], i.a, i.skip,
                                           i.bias, True)
            _inside(got[0][r].view(d, n), h, err, None, f"state {e}")
            _inside(out[c0:c1], y, bound, dt, f"rows {e}")
        assert (out[20:60] == 7).all()
    else:
        call([1, 3], [0, 20, 20], want)
        call([3], [60, tot], want)
        assert torch.equal(out, want)
        ref = _states(ctx, 0, [1, 2, 3, 4, 5], m)
        if op == "conv":       # slot 3 went through two calls above: without rows its window stays as it was
            assert torch.equal(got[1], ref[1])
        else:
            assert torch.equal(got[0], ref[0])
    for e in (1, 3, 4):
        assert torch.equal(got[0][e], st[e]) and torch.equal(got[1][e], cv[e])
    ctx.close()


@pytest.mark.gpu
def test_refusals_of_conv_and_scan():
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = torch.bfloat16
    d, n, w = 64, 16, 4
    ctx = _ctx(_model(d, n, w), 8, [0, 1])
    x = torch.zeros(8, 8 * d, dtype=dt, device="cuda")
    f = torch.zeros(4096, device="cuda")
    ok = dict(channels=d, width=w, silu=True, dtype=dt)

    def conv(layer=0, n=2, xx=x, weight=f, bias=f, out=x, total=8, **kw):
        desc = B.conv_desc(**{**ok, **kw})
        ctx.conv_prompt(layer, desc, _i32([0, 1]), n, _i32([0, 1, 2]), total, None, xx, weight, bias, out)
        ctx.conv_step(layer, desc, _i32([0, 1]), n, xx, weight, bias, out)

    conv(out=torch.zeros_like(x))
    for bad in (dict(layer=2), dict(n=9), dict(channels=d + 8), dict(width=3), dict(width=5, channels=48), dict(channels=0), dict(x_stride_bytes=8),
                dict(x_stride_bytes=d * 2 + 8), dict(out_stride_bytes=16), dict(xx=None), dict(xx=x[:, 4:]), dict(weight=None), dict(weight=f[1:]),
                dict(bias=f[2:]), dict(out=x[:, 1:])):
        with pytest.raises(B.AvmpError):
            conv(**bad)
    sok = dict(channels=d, groups=1, states=n, softplus=True, dtype=dt)

    def scan(layer=0, n=2, u=x, z=x, a=f, skip=f, bias=f, out=x, **kw):
        desc = B.scan_desc(**{**sok, **kw})
        ctx.scan_prompt(layer, desc, _i32([0, 1]), n, _i32([0, 1, 2]), 8, None, u, x, x, x, z, a, skip, bias, out)
        ctx.scan_step(layer, desc, _i32([0, 1]), n, u, x, x, x, z, a, skip, bias, out)

    scan(out=torch.zeros_like(x))
    for bad in (dict(layer=2), dict(n=9), dict(channels=2 * d), dict(states=32), dict(states=12), dict(groups=3), dict(groups=0), dict(groups=16),
                dict(u_stride_bytes=24), dict(b_stride_bytes=16), dict(z_stride_bytes=d * 2 - 16), dict(out_stride_bytes=d * 2 + 4), dict(u=None),
                dict(u=x[:, 3:]), dict(z=x[:, 1:]), dict(a=None), dict(a=f[1:]), dict(out=None)):
        with pytest.raises(B.AvmpError):
            scan(**bad)
    with pytest.raises(B.AvmpError):
        B.scan_desc(**{**sok, "dtype": torch.float32})
    with pytest.raises(B.AvmpError):
        B.conv_desc(**{**ok, "dtype": torch.float32})
    # a long prompt of few channels needs its scratch
    desc = B.scan_desc(**sok)
    size = ctx.scan_workspace_bytes(desc, 1, 5000)
    assert size > 0 and ctx.scan_workspace_bytes(desc, 0, 5000) == 0 and ctx.scan_workspace_bytes(B.scan_desc(**{**sok, "states": 32}), 1, 5000) == 0
    rows = torch.zeros(5000, d, dtype=dt, device="cuda")
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    for w_, s_ in ((None, size), (ws, size - 1), (ws[1:], size)):
        with pytest.raises(B.AvmpError):
            ctx.scan_prompt(0, desc, _i32([0]), 1, _i32([0, 5000]), 5000, None, rows, rows, rows, rows, None, f, None, None, torch.empty_like(rows),
                            w_, s_)
    assert ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
def test_nonfinite_numbers_stay_in_their_channel():
    """A NaN in a channel's input, an infinity in another's state: these channels' states are lost, the other channels, groups and requests are not
    touched.  Rows behind the last and in front of a request hold NaN throughout."""
    import torch
    dt = torch.float16
    d, g, n = 64, 2, 16
    m = _model(d, n, 2, layers=1)
    ctx = _ctx(m, 4, [0, 1])
    gen = torch.Generator("cuda").manual_seed(1)
    st, cv = _fill(ctx, 0, [0, 1], m, gen, dt)
    tot = 100
    i = _scan_inputs(d, g, n, tot, dt, gen)
    for x in (i.u, i.delta, i.z, i.b, i.c):
        x[:10] = math.nan
        x[80:] = math.nan
    desc = _scan_desc(i, d, g, n, dt)
    out = torch.full((tot, d), 7.0, dtype=dt, device="cuda")
    args = lambda: (i.u, i.delta, i.b, i.c, i.z, i.a, i.skip, i.bias)
    cu = _i32([10, 45, 80])
    ctx.scan_prompt(0, desc, _i32([0, 1]), 2, cu, tot, _i32([1, 1]), *args(), out)
    ref, ref_st = out.clone(), _states(ctx, 0, [0, 1], m)[0]
    assert torch.isfinite(out).all() and (out[:10] == 7).all() and (out[80:] == 7).all() and torch.isfinite(ref_st).all()
    bad = st.clone()
    bad[1].view(d, n)[40, 3] = math.inf
    ctx.scatter_ssm(0, _i32([0, 1]), 2, bad, cv)
    i.u[20, 5] = math.nan
    ctx.scan_prompt(0, desc, _i32([0, 1]), 2, cu, tot, _i32([1, 1]), *args(), out)
    got = _states(ctx, 0, [0, 1], m)[0].view(2, d, n)
    keep = torch.ones(2, d, dtype=torch.bool, device="cuda")
    keep[0, 5] = keep[1, 40] = False
    assert torch.equal(got[keep], ref_st.view(2, d, n)[keep]) and not torch.isfinite(got[0, 5]).any() and not torch.isfinite(got[1, 40, 3])
    assert torch.isfinite(got[1, 40, :3]).all()
    assert torch.equal(out[10:45][:, keep[0]], ref[10:45][:, keep[0]]) and torch.equal(out[45:80][:, keep[1]], ref[45:80][:, keep[1]])
    assert torch.equal(out[10:20, 5], ref[10:20, 5]) and torch.isnan(out[20:45, 5]).all()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("d", [16, 2048])
def test_masked_steps(dtype, d):
    """Tokens whose step is masked, by the type's lowest value or minus infinity, leave the state as it was; a step of NaN does not pass for one."""
    import torch
    dt = getattr(torch, dtype)
    n = 16
    m = _model(d, n, 2, layers=1)
    ctx = _ctx(m, 4, [0, 1, 2])
    gen = torch.Generator("cuda").manual_seed(d)
    st, cv = _fill(ctx, 0, [0, 1, 2], m, gen, dt)
    tot = 70
    i = _scan_inputs(d, 1, n, tot, dt, gen)
    i.delta[:, ::2] = -math.inf
    i.delta[:, 1::2] = torch.finfo(dt).min
    out = torch.empty(tot, d, dtype=dt, device="cuda")
    desc = _scan_desc(i, d, 1, n, dt)
    args = lambda: (i.u, i.delta, i.b, i.c, i.z, i.a, i.skip, i.bias)
    ctx.scan_prompt(0, desc, _i32([0, 1]), 2, _i32([0, 69, 70]), tot, _i32([1, 1]), *args(), out)
    ctx.scan_step(0, desc, _i32([2]), 1, *args(), out)
    assert torch.equal(_states(ctx, 0, [0, 1, 2], m)[0], st) and torch.isfinite(out).all()
    h, _, y, bound = _scan_exact(st[2].view(d, n), i.u[:1], torch.full_like(i.delta[:1], -1000.0), i.b[:1, None], i.c[:1, None], i.z[:1], i.a, i.skip, i.bias,
                                 True)
    _inside(out[:1], y, bound, dt, "a masked token's output")
    i.delta[3, 5] = math.nan
    ctx.scan_prompt(0, desc, _i32([0, 1]), 2, _i32([0, 69, 70]), tot, _i32([1, 1]), *args(), out)
    got = _states(ctx, 0, [0], m)[0].view(d, n)
    assert torch.isnan(got[5]).all() and torch.equal(got[:5], st[0].view(d, n)[:5]) and torch.isnan(out[3:69, 5]).all() and torch.isfinite(out[:3]).all()
    ctx.close()


@pytest.mark.gpu
def test_calls_without_rows():
    """No rows at all, no buffers: fresh requests get zeros, continued ones keep what they have."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = torch.bfloat16
    d, n, w = 40, 8, 3
    m = _model(d, n, w, layers=1)
    ctx = _ctx(m, 4, [0, 1])
    gen = torch.Generator("cuda").manual_seed(1)
    st, cv = _fill(ctx, 0, [0, 1], m, gen, dt)
    f = torch.zeros(d * n, device="cuda")
    none = [None] * 5
    ctx.conv_prompt(0, B.conv_desc(channels=d, width=w, silu=True, dtype=dt), _i32([0, 1]), 2, _i32([0, 0, 0]), 0, _i32([1, 0]), None, f, None, None)
    ctx.scan_prompt(0, B.scan_desc(channels=d, groups=1, states=n, softplus=True, dtype=dt), _i32([0, 1]), 2, _i32([0, 0, 0]), 0, _i32([1, 0]), *none, f,
                    None, None, None)
    st2, cv2 = _states(ctx, 0, [0, 1], m)
    assert torch.equal(st2[0], st[0]) and torch.equal(cv2[0], cv[0]) and not st2[1].any() and not cv2[1].any()
    assert ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
def test_long_lists_and_offsets():
    """More entries than a CTA has threads, with repeated slots: the first of each stands."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = torch.bfloat16
    d, n, w = 16, 8, 4
    slots = 700
    m = _model(d, n, w, layers=1)
    ctx = _ctx(m, slots, range(slots))
    gen = torch.Generator("cuda").manual_seed(2)
    st, cv = _fill(ctx, 0, range(slots), m, gen, dt)
    rng = np.random.default_rng(3)
    reqs = rng.permutation(slots)
    reqs[[300, 699]] = reqs[[5, 298]]
    lens = rng.integers(0, 20, slots)
    cu = np.concatenate([[0], np.cumsum(lens)])
    tot = int(cu[-1])
    i = _scan_inputs(d, 1, n, tot, dt, gen)
    out, conv_out = (torch.full((tot, d), 7.0, dtype=dt, device="cuda") for _ in range(2))
    weight = torch.randn(d, w, device="cuda", generator=gen)
    ctx.conv_prompt(0, B.conv_desc(channels=d, width=w, silu=True, dtype=dt, x_stride_bytes=i.us), _i32(reqs), slots, _i32(cu), tot, _i32([1] * slots),
                    i.u, weight, None, conv_out)
    ctx.scan_prompt(0, _scan_desc(i, d, 1, n, dt), _i32(reqs), slots, _i32(cu), tot, _i32([1] * slots), i.u, i.delta, i.b, i.c, i.z, i.a, i.skip, i.bias,
                    out)
    st2, cv2 = _states(ctx, 0, range(slots), m)
    for e in (0, 5, 128, 255, 298, 300, 511, 698, 699):
        r, sl = int(reqs[e]), slice(cu[e], cu[e + 1])
        if e in (300, 699):
            assert (out[sl] == 7).all() and (conv_out[sl] == 7).all()
            continue
        h, err, y, bound = _scan_exact(st[r].view(d, n), i.u[sl], i.delta[sl], i.b[sl, None], i.c[sl, None], i.z[sl], i.a, i.skip, i.bias, True)
        _inside(st2[r].view(d, n), h, err, None, f"state {e}")
        _inside(out[sl], y, bound, dt, f"rows {e}")
        y, bound, new = _conv_exact(i.u[sl], cv[r].view(w - 1, d), weight, None, True)
        _inside(conv_out[sl], y, bound, dt, f"convolution of {e}")
        assert torch.equal(cv2[r].view(w - 1, d).double(), new)
    assert ctx.stats()["error_count"] == 4
    ctx.close()


@pytest.mark.gpu
def test_prompts_in_a_graph():
    """Convolution and a scan cut into runs, captured together and replayed on another stream: the same, bit for bit, as the calls made one by one;
    continued from where the replay before ended."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = torch.bfloat16
    d, n, w, tot = 64, 16, 4, 2000
    m = _model(d, n, w, layers=1)
    ctx = _ctx(m, 4, [0, 2])
    gen = torch.Generator("cuda").manual_seed(9)
    st, cv = _fill(ctx, 0, [0, 2], m, gen, dt)
    i = _scan_inputs(d, 1, n, tot, dt, gen)
    weight = torch.randn(d, w, device="cuda", generator=gen)
    conv = B.conv_desc(channels=d, width=w, silu=True, dtype=dt, x_stride_bytes=i.us)
    scan = B.scan_desc(channels=d, groups=1, states=n, softplus=True, dtype=dt, delta_stride_bytes=i.ds, z_stride_bytes=i.zs, b_stride_bytes=i.bs,
                       c_stride_bytes=i.bs)
    size = ctx.scan_workspace_bytes(scan, 2, tot)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    reqs, cu, resume = _i32([2, 0]), _i32([0, 1500, tot]), _i32([1, 1])
    mid, out = (torch.empty(tot, d, dtype=dt, device="cuda") for _ in range(2))

    def both():
        ctx.conv_prompt(0, conv, reqs, 2, cu, tot, resume, i.u, weight, None, mid)
        ctx.scan_prompt(0, scan, reqs, 2, cu, tot, resume, mid, i.delta, i.b, i.c, i.z, i.a, i.skip, i.bias, out, ws, size)

    want = []
    for _ in range(2):
        both()
        want.append((mid.clone(), out.clone(), *_states(ctx, 0, [0, 2], m)))
    ctx.scatter_ssm(0, _i32([0, 2]), 2, st, cv)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for k in range(2):
        mid.zero_(), out.zero_(), ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((mid, out, *_states(ctx, 0, [0, 2], m)), want[k])), k
    assert ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,states,tot", [(197, 32, 16, 197 * 384), (151, 24, 8, 58086), (167, 8, 16, 64246), (98, 32, 16, 98 * 800)])
def test_scratch_of_many_requests_that_are_cut(n, d, states, tot):
    """Many requests (at times more than SMs), each cut into runs: the call stays within the scratch that the query asks for."""
    import torch
    dt = torch.bfloat16
    m = _model(d, states, 4, layers=1)
    ctx = _ctx(m, n, range(n))
    gen = torch.Generator("cuda").manual_seed(n)
    st, _ = _fill(ctx, 0, range(n), m, gen, dt)
    i = _scan_inputs(d, 1, states, tot, dt, gen)
    desc = _scan_desc(i, d, 1, states, dt)
    size, guard = ctx.scan_workspace_bytes(desc, n, tot), 1 << 20
    assert size > 0
    ws = torch.full((size + guard,), 0x5A, dtype=torch.uint8, device="cuda")
    cu = np.linspace(0, tot, n + 1).astype(np.int64)
    out = torch.empty(tot, d, dtype=dt, device="cuda")
    ctx.scan_prompt(0, desc, _i32(range(n)), n, _i32(cu), tot, _i32([1] * n), i.u, i.delta, i.b, i.c, i.z, i.a, i.skip, i.bias, out, ws, size)
    st2, _ = _states(ctx, 0, range(n), m)
    assert (ws[size:] == 0x5A).all()
    for e in (0, n - 1):
        r = slice(cu[e], cu[e + 1])
        h, err, y, bound = _scan_exact(st[e].view(d, states), i.u[r], i.delta[r], i.b[r, None], i.c[r, None], i.z[r], i.a, i.skip, i.bias, True)
        _inside(st2[e].view(d, states), h, err, None, f"state {e}")
        _inside(out[r], y, bound, dt, f"rows of {e}")
    assert ctx.stats()["error_count"] == 0
    ctx.close()
