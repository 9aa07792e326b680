"""Selective scan where decays, states or rows reach the ends of the 32-bit range, and what a missing row means there."""
from __future__ import annotations

import math

import numpy as np
import pytest

from test_conv_scan import _fill, _inside, _model, _scan_exact, _scan_inputs
from test_ssm_ops import _ctx, _i32, _states


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,d", [(1, 16), (20, 256)])
def test_decay_of_a_whole_run_passes_the_range(dtype, n, d):
    """Prompts that are cut into runs, with steps of 1 for 80 tokens, 0 for the others: the product of a run's decays is e^(80 A), as much as 2^173 or
    as little as 2^-173.  States are what they are token by token: zeros stay zeros, infinities infinities, and small or large ones come into or stay
    within the range.  Inputs are zero, so that nothing is added."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt, states, most = getattr(torch, dtype), 16, 3000 if n == 1 else 500
    m = _model(d, states, 2, layers=1)
    ctx = _ctx(m, n, range(n))
    gen = torch.Generator("cuda").manual_seed(d)
    st, cv = _fill(ctx, 0, range(n), m, gen, dt)
    a = torch.full((d, states), 0.25, device="cuda")
    a[:, 1::4], a[:, 2::4], a[:, 3::4] = -0.25, 1.5, -1.5
    st = st.view(n, d, states)
    st[:, 0::4] = 0
    st[:, 1::4] = math.inf
    st[:, 2::4, 2::4] *= 1e-30                          # times 2^173: within the range again
    st[:, 2::4, 3::4] *= 1e30                           # times 2^-173: still within it
    st[:, 3::4, 2::4], st[:, 3::4, 3::4] = 1e20, 1e-20  # out of it, at either end
    ctx.scatter_ssm(0, _i32(range(n)), n, st.reshape(n, -1), cv)
    tot = n * most
    step = torch.zeros(tot, d, dtype=dt, device="cuda")
    for e in range(n):
        step[e * most + 5: e * most + 85] = 1           # (in the first of the runs, which take 128 tokens or more)
    zeros = torch.zeros(tot, d, dtype=dt, device="cuda")
    bc = torch.randn(tot, 2 * states, device="cuda", generator=gen).to(dt)
    desc = B.scan_desc(channels=d, groups=1, states=states, softplus=False, dtype=dt, b_stride_bytes=4 * states, c_stride_bytes=4 * states)
    size = ctx.scan_workspace_bytes(desc, n, tot)
    assert size > 0
    ws, out = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda"), torch.empty(tot, d, dtype=dt, device="cuda")
    ctx.scan_prompt(0, desc, _i32(range(n)), n, _i32(np.arange(n + 1) * most), tot, _i32([1] * n), zeros, step, bc, bc[:, states:], None, a, None, None,
                    out, ws, size)
    got = _states(ctx, 0, range(n), m)[0].view(n, d, states)
    want = st.double() * (80 * a.double()).exp()
    # 80 exponentials, their argument's roundings, the sum of steps, a rounding a token; and once more of the product of decays, in four parts
    bound = want.abs() * (80 * 2.0 ** -22 + 80 * a.double().abs() * 2.0 ** -21 + (80 + 8) * 2.0 ** -23) + 2.0 ** -126
    assert (got[:, 0::4] == 0).all() and (got[:, 1::4] == math.inf).all()
    large = torch.isfinite(want) & (want.abs() > torch.finfo(torch.float32).max)
    assert (got[large] == math.inf).all() and large.any()
    rest = torch.isfinite(want) & ~large
    assert float(((got.double() - want).abs() - bound)[rest].max()) <= 0
    assert (want[:, 2::4, 3::4].abs() > 1e-30).any()
    assert (out[:, 0::4] == 0).all() and ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states", [8, 16, 64])
def test_infinite_rows_without_the_skip_term(states):
    """Without D an infinite row is seen through the state alone, by single tokens as by prompts: there is no 0 * infinity."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt, d = torch.bfloat16, 40
    m = _model(d, states, 2, layers=1)
    ctx = _ctx(m, 2, [0, 1])
    gen = torch.Generator("cuda").manual_seed(states)
    st, cv = _fill(ctx, 0, [0, 1], m, gen, dt)
    st[1] = st[0]
    ctx.scatter_ssm(0, _i32([0, 1]), 2, st, cv)
    u, delta = (torch.randn(1, d, device="cuda", generator=gen).to(dt) for _ in range(2))
    b, c = (torch.rand(1, states, device="cuda", generator=gen).to(dt) + 0.5 for _ in range(2))
    u[0, 3], u[0, 17], u[0, 39] = math.inf, -math.inf, math.inf
    a = -torch.rand(d, states, device="cuda", generator=gen) - 0.1
    desc = B.scan_desc(channels=d, groups=1, states=states, softplus=True, dtype=dt)
    outs = [torch.empty(1, d, dtype=dt, device="cuda") for _ in range(2)]
    ctx.scan_prompt(0, desc, _i32([0]), 1, _i32([0, 1]), 1, _i32([1]), u, delta, b, c, None, a, None, None, outs[0])
    ctx.scan_step(0, desc, _i32([1]), 1, u, delta, b, c, None, a, None, None, outs[1])
    hit = torch.isinf(u[0])
    got, _ = _states(ctx, 0, [0, 1], m)
    for o, h in zip(outs, got.view(2, d, states)):
        assert torch.equal(o[0, hit].float(), u[0, hit].float()) and torch.equal(h[hit], u[0, hit].float()[:, None].expand(-1, states))
        hh, err, y, bound = _scan_exact(st[0].view(d, states)[~hit], u[:, ~hit], delta[:, ~hit], b[:, None], c[:, None], None, a[~hit], None, None, True)
        _inside(o[:, ~hit], y, bound, dt, "the others")
        _inside(h[~hit], hh, err, None, "the others' states")
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("call", ["prompt", "step"])
def test_mean_error_of_a_decay(call):
    """What a state loses or gains by one token's decay, on the mean over a million states: a part of 5e-9 at most for exponents of 2^-13 to 2^-9 (the
    instruction by itself 6e-9 too little), 1.8e-8 for 2^-7.5 to 2^-1 (by itself 2.1e-8 too little).  A rounding of the state is 3e-8 at most and to
    either side: 3e-11 on the mean."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt, d, states, n = torch.bfloat16, 4096, 16, 16
    m = _model(d, states, 2, layers=1)
    ctx = _ctx(m, n, range(n))
    gen = torch.Generator("cuda").manual_seed(3)
    zeros, ones = torch.zeros(n, d, dtype=dt, device="cuda"), torch.ones(n, d, dtype=dt, device="cuda")
    bc, out = torch.ones(n, states, dtype=dt, device="cuda"), torch.empty(n, d, dtype=dt, device="cuda")
    desc = B.scan_desc(channels=d, groups=1, states=states, softplus=False, dtype=dt)
    ws, size = torch.empty(max(16, ctx.scan_workspace_bytes(desc, n, n)), dtype=torch.uint8, device="cuda"), ctx.scan_workspace_bytes(desc, n, n)
    for lo, hi, most in ((-13.0, -9.0, 5e-9), (-7.5, -1.0, 1.8e-8)):
        a = -torch.exp2(lo + (hi - lo) * torch.rand(d, states, device="cuda", generator=gen)) * math.log(2)
        st = torch.rand(n, d, states, device="cuda", generator=gen) + 0.5
        ctx.scatter_ssm(0, _i32(range(n)), n, st.reshape(n, -1), torch.zeros(n, m.ssm_conv_elems, device="cuda"))
        rows = (zeros, ones, bc, bc, None, a, None, None, out)
        if call == "prompt":
            ctx.scan_prompt(0, desc, _i32(range(n)), n, _i32(range(n + 1)), n, _i32([1] * n), *rows, ws, size)
        else:
            ctx.scan_step(0, desc, _i32(range(n)), n, *rows)
        want = st.double() * a.double().exp()
        off = float(((_states(ctx, 0, range(n), m)[0].view(n, d, states).double() - want) / want).mean())
        assert abs(off) <= most, (lo, hi, off)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,most", [(300, 2.5e-6), (20000, 6e-5)])
def test_slow_states_on_the_mean(tokens, most):
    """States that remember `tokens` tokens (0.7 to 1.4 times as many), fed with ones: on the mean they are off by the decays' mean error as many
    times, 3e-9 at most where that is 20 000, 8e-9 for 300."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt, d, states, total = torch.bfloat16, 4096, 16, tokens * 2
    m = _model(d, states, 2, layers=1)
    ctx = _ctx(m, 1, [0])
    a = -1 / torch.linspace(0.7 * tokens, 1.4 * tokens, d * states, device="cuda").view(d, states)
    ones, bc = torch.ones(total, d, dtype=dt, device="cuda"), torch.ones(total, states, dtype=dt, device="cuda")
    desc = B.scan_desc(channels=d, groups=1, states=states, softplus=False, dtype=dt)
    size = ctx.scan_workspace_bytes(desc, 1, total)
    ws = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")
    ctx.scan_prompt(0, desc, _i32([0]), 1, _i32([0, total]), total, None, ones, ones, bc, bc, None, a, None, None, torch.empty_like(ones), ws, size)
    decay = a.double().exp()
    want = (1 - decay ** total) / (1 - decay)
    off = float(((_states(ctx, 0, [0], m)[0].view(d, states).double() - want) / want).mean())
    assert abs(off) <= most, off
    ctx.close()
