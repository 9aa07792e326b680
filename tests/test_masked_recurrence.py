"""The recurrence on the SSM state blocks where rows must not count (tokens behind a row, tokens in front of a reset), bounds
entry by entry, and states that are carried over the runs that a long prompt is cut into.

Tolerances.  An output is sum over tokens and dk of terms e^(..) v k q.  Rounded to 16 bits are the decayed scores, the carried
state as an operand, and the output: 3 * eps/2 of the sum of the terms' absolute values (which the same recurrence on absolute
values gives); exponents of up to 600 in log2 units are good to 2^-15, and that with the 32-bit sums stays inside a quarter
of eps/2.  The state: e^(..) v enters with 22 bits (fp16, two parts) or 24 (bf16, three), exponentials are good to 2^-22, one to a
term and one more for each piece of 64 tokens it is carried over: (pieces + 2) * 2^-22 norm-wise."""
from __future__ import annotations

import math

import numpy as np
import pytest

from test_ssm_ops import _ctx, _fill_state, _i32, _model, _states


def _recurrence(S, q, k, v, g, rep):
    """64 bits, token by token: state, outputs, and the outputs of the absolute values.  S [heads, dv, dk]."""
    import torch
    out = torch.zeros(v.shape, dtype=torch.float64, device=v.device)
    size, A = torch.zeros_like(out), S.abs()
    q, k = (x.double().repeat_interleave(rep, 1) for x in (q, k))
    v, g = v.double(), g.double()
    for t in range(v.shape[0]):
        w = g[t].exp()[:, None, None]
        vk = v[t][:, :, None] * k[t][:, None, :]
        S = torch.where(w == 0, vk, S * w + vk)
        A = torch.where(w == 0, vk.abs(), A * w + vk.abs())
        out[t] = (S * q[t][:, None, :]).sum(-1)
        size[t] = (A * q[t][:, None, :].abs()).sum(-1)
    return S, out, size


def _near(out, want, size, what):
    """Finite where the definition is, and close there."""
    import torch
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(out), fin), f"{what}: {int((torch.isfinite(out) != fin).sum())} entries finite or not where they should be"
    # An output below the type's normal range is rounded by half the spacing there, smallest_normal * eps, and not by eps/2 of itself.
    info = torch.finfo(out.dtype)
    d = ((out.double() - want).abs() - 3.25 * info.eps / 2 * size - info.smallest_normal * info.eps / 2)[fin]
    assert d.numel() == 0 or float(d.max()) <= 0, f"{what}: {float(d.max()):.3g} too far off"


def _near_state(got, want, pieces, what):
    import torch
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fin), f"{what}: {int((torch.isfinite(got) != fin).sum())} entries finite or not where they should be"
    err = float(((got.double() - want)[fin]).norm() / want[fin].norm().clamp(min=1e-300))
    assert err <= (pieces + 2) * 2.0 ** -22, f"{what}: relative error {err:.3g}"


SHAPES = [(2, 1, 16, 64), (3, 1, 16, 32), (4, 2, 32, 64), (2, 2, 64, 96), (2, 1, 128, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("what", ["v", "k", "state", "decay"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_a_bad_row_counts_from_itself_to_the_next_reset(shape, what, value, dtype):
    import torch
    from paper_2605_22416_b200 import binding as B
    if what == "decay" and not math.isnan(value):
        return                                          # decays are at most 0, and -inf is the reset
    heads, groups, dk, dv = SHAPES[shape]
    dt, m = getattr(torch, dtype), _model(heads, dk, dv)
    lens, n = [300, 90, 64], 3
    tot, cu = sum(lens), np.concatenate([[0], np.cumsum(lens)])
    ctx = _ctx(m, 4, [0, 1, 2])
    gen = torch.Generator("cuda").manual_seed(shape)
    first, conv = _fill_state(ctx, 1, [0, 1, 2], m, gen, scale=0.5)
    q, k = ((torch.randn(tot, groups, dk, device="cuda", generator=gen) * 0.3).to(dt) for _ in range(2))
    v = torch.randn(tot, heads, dv, device="cuda", generator=gen).to(dt)
    g = -torch.rand(tot, heads, device="cuda", generator=gen) ** 4 * 0.2
    # request 0: bad at 21 (reset at 30, in the next block of 16), at 40 (reset at 44, in its own), at 70 (reset a piece later),
    # at 200 of one head's row (never reset); request 1: bad at 10, reset in head 0 only; request 2: clean
    bad, resets = [21, 40, 70, 200, cu[1] + 10], [30, 44, 140, cu[1] + 15]
    for t in resets:
        g[t, 0 if t > cu[1] else slice(None)] = -math.inf
    if what == "v":
        for i, t in enumerate(bad):
            v[t, i % heads, 3 * i + 1] = value
    elif what == "k":
        for i, t in enumerate(bad):
            k[t, i % groups, (5 * i + 2) % dk] = value
    elif what == "decay":
        for t in bad:
            g[t, heads - 1] = value
    else:
        st = first.view(n, heads, dv, dk)
        st[0, 0, 5, 3], st[1, 0, 7, 1], st[1, heads - 1, dv - 1, dk - 1] = value, value, value
        ctx.scatter_ssm(1, _i32([0, 1, 2]), n, first, conv)
    desc = B.ssm_desc(heads=heads, groups=groups, dk=dk, dv=dv, dtype=dt)
    out = torch.zeros_like(v)
    ctx.ssm_prompt(1, desc, _i32([0, 1, 2]), n, _i32(cu), tot, _i32([1, 1, 0]), q, k, v, g, out)
    st, cv = _states(ctx, 1, [0, 1, 2], m)
    for r in range(n):
        a, b = cu[r], cu[r + 1]
        S0 = first[r].view(heads, dv, dk).double() if r < 2 else torch.zeros(heads, dv, dk, dtype=torch.float64, device="cuda")
        S, o, _ = _recurrence(S0, q[a:b], k[a:b], v[a:b], g[a:b], heads // groups)
        z = lambda x: torch.nan_to_num(x, 0.0, 0.0, -math.inf if x is g else 0.0)        # sizes without the bad entries
        size = _recurrence(z(S0), z(q)[a:b], z(k)[a:b], z(v)[a:b], z(g)[a:b], heads // groups)[2]
        _near(out[a:b], o, size, f"request {r}")
        _near_state(st[r].view(heads, dv, dk), S, -(-lens[r] // 64), f"state {r}")
        if r < 2:
            assert torch.isfinite(o).any() and not torch.isfinite(o).all()
    assert torch.equal(cv, conv) and ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("heads,groups,dk,dv,lens", [(4, 2, 16, 64, [300, 17]), (2, 1, 32, 96, [250]), (2, 1, 64, 64, [200, 65]), (2, 2, 128, 32, [130])])
def test_entry_by_entry(dtype, heads, groups, dk, dv, lens):
    """Finite rows: every output by itself, and states to the precision that three (two) 16-bit parts of e^(..) v give."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt, m, n, tot = getattr(torch, dtype), _model(heads, dk, dv), len(lens), sum(lens)
    cu = np.concatenate([[0], np.cumsum(lens)])
    ctx = _ctx(m, 4, list(range(n)))
    gen = torch.Generator("cuda").manual_seed(dk + dv)
    q, k = ((torch.randn(tot, groups, dk, device="cuda", generator=gen) * 0.3).to(dt) for _ in range(2))
    v = torch.randn(tot, heads, dv, device="cuda", generator=gen).to(dt)
    g = -torch.rand(tot, heads, device="cuda", generator=gen) ** 4 * 0.2
    out = torch.zeros_like(v)
    ctx.ssm_prompt(0, B.ssm_desc(heads=heads, groups=groups, dk=dk, dv=dv, dtype=dt), _i32(range(n)), n, _i32(cu), tot, None, q, k, v, g, out)
    st, _ = _states(ctx, 0, list(range(n)), m)
    for r in range(n):
        a, b = cu[r], cu[r + 1]
        S, o, size = _recurrence(torch.zeros(heads, dv, dk, dtype=torch.float64, device="cuda"), q[a:b], k[a:b], v[a:b], g[a:b], heads // groups)
        _near(out[a:b], o, size, f"request {r}")
        _near_state(st[r].view(heads, dv, dk), S, -(-lens[r] // 64), f"state {r}")
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,heads,dk,dv,lens", [("bfloat16", 1, 16, 64, [4000]), ("float16", 2, 64, 32, [33, 6000]), ("bfloat16", 3, 128, 64, [4097])])
def test_states_carried_over_the_runs_of_a_cut_prompt(dtype, heads, dk, dv, lens):
    """Decays so gentle that the state in the block and every earlier run count visibly in the last one."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt, m, n, tot = getattr(torch, dtype), _model(heads, dk, dv), len(lens), sum(lens)
    cu = np.concatenate([[0], np.cumsum(lens)])
    ctx = _ctx(m, 4, list(range(n)))
    gen = torch.Generator("cuda").manual_seed(dk)
    first, _ = _fill_state(ctx, 1, list(range(n)), m, gen, scale=30.0)
    q, k = ((torch.randn(tot, 1, dk, device="cuda", generator=gen) * 0.2).to(dt) for _ in range(2))
    v = torch.randn(tot, heads, dv, device="cuda", generator=gen).to(dt)
    g = -torch.rand(tot, heads, device="cuda", generator=gen) * 2e-4
    desc = B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=dt)
    size = ctx.ssm_workspace_bytes(desc, n, tot)
    assert size > 0
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(v)
    ctx.ssm_prompt(1, desc, _i32(range(n)), n, _i32(cu), tot, _i32([1] * n), q, k, v, g, out, ws, size)
    st, _ = _states(ctx, 1, list(range(n)), m)
    for r in range(n):
        a, b = cu[r], cu[r + 1]
        S, o, mass = _recurrence(first[r].view(heads, dv, dk).double(), q[a:b], k[a:b], v[a:b], g[a:b], heads)
        _near(out[a:b], o, mass, f"request {r}")
        _near_state(st[r].view(heads, dv, dk), S, -(-lens[r] // 64), f"state {r}")
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("heads,dk,dv", [(32, 16, 64), (1, 128, 32), (8, 64, 96)])
def test_a_workspace_for_the_largest_batch_serves_smaller_ones(heads, dk, dv):
    import torch
    from paper_2605_22416_b200 import binding as B
    m, slots = _model(heads, dk, dv, layers=1), 34
    ctx = _ctx(m, slots, list(range(slots)))
    desc = B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=torch.bfloat16)
    most, total = slots, 4000
    sizes = [[ctx.ssm_workspace_bytes(desc, n, t) for t in (0, 1, 500, 2000, 3999, total)] for n in range(1, most + 1)]
    assert all(a <= b for row in sizes for a, b in zip(row, row[1:])) and all(a <= b for x, y in zip(sizes, sizes[1:]) for a, b in zip(x, y))
    size = sizes[-1][-1]
    assert 0 < size < 5 << 20
    ws = torch.full((size + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    gen = torch.Generator("cuda").manual_seed(heads)
    q, k = ((torch.randn(total, 1, dk, device="cuda", generator=gen) * 0.2).to(torch.bfloat16) for _ in range(2))
    v = torch.randn(total, heads, dv, device="cuda", generator=gen).to(torch.bfloat16)
    g = -torch.rand(total, heads, device="cuda", generator=gen) * 1e-2
    for n, tot in ((1, 2500), (2, 4000), (most, total)):
        cu = np.linspace(0, tot, n + 1).astype(int)
        out = torch.zeros_like(v)
        ctx.ssm_prompt(0, desc, _i32(range(n)), n, _i32(cu), tot, None, q, k, v, g, out, ws, size)
        r = n - 1
        _, o, mass = _recurrence(torch.zeros(heads, dv, dk, dtype=torch.float64, device="cuda"), *(x[cu[r]:cu[r + 1]] for x in (q, k, v, g)), heads)
        _near(out[cu[r]:cu[r + 1]], o, mass, f"{n} requests")
    out = torch.zeros_like(v)
    ctx.ssm_prompt(0, desc, _i32(range(most)), most, _i32(np.linspace(0, total, most + 1).astype(int)), total, None, q, k, v, g, out)      # not cut: no workspace
    assert (ws[size:] == 0xFF).all() and ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(1 << 22) + 1, (1 << 23) - 1])
def test_blocks_too_large_to_count_are_refused(heads):
    """More than 2^31 state elements (no such block fits this pool; the call is refused before it looks)."""
    import torch
    from paper_2605_22416_b200 import binding as B
    ctx = B.Context(_model(heads, 16, 32), 1 << 20, 0.0, 1, max_requests=2, max_pages=4)
    desc = B.ssm_desc(heads=heads, groups=1, dk=16, dv=32, dtype=torch.bfloat16)
    x = torch.zeros(1024, device="cuda")
    with pytest.raises(B.AvmpError, match="invalid argument"):
        ctx.ssm_step(0, desc, _i32([0]), 1, x, x, x, x, x)
    with pytest.raises(B.AvmpError, match="invalid argument"):
        ctx.ssm_prompt(0, desc, _i32([0]), 1, _i32([0, 1]), 1, None, x, x, x, x, x)
    assert ctx.ssm_workspace_bytes(desc, 1, 1 << 20) == 0 and ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("heads,dk,dv", [(1, 16, 64), (2, 128, 32)])
def test_bad_rows_in_a_cut_prompt(heads, dk, dv, value, dtype):
    """The same over the runs of a long prompt: a bad state in the block, reset in the first run; a bad row in one run, reset in a
    later one; a bad row that is never reset."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt, m, tot = getattr(torch, dtype), _model(heads, dk, dv), 4000
    ctx = _ctx(m, 2, [0])
    gen = torch.Generator("cuda").manual_seed(dk)
    first, conv = _fill_state(ctx, 0, [0], m, gen)
    first.view(heads, dv, dk)[0, 3, 5] = value
    ctx.scatter_ssm(0, _i32([0]), 1, first, conv)
    q, k = ((torch.randn(tot, 1, dk, device="cuda", generator=gen) * 0.2).to(dt) for _ in range(2))
    v = torch.randn(tot, heads, dv, device="cuda", generator=gen).to(dt)
    g = -torch.rand(tot, heads, device="cuda", generator=gen) * 1e-3
    g[[300, 2900]] = -math.inf
    v[900, heads - 1, 7], v[3300, 0, 20] = value, value
    desc = B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=dt)
    size = ctx.ssm_workspace_bytes(desc, 1, tot)
    assert size > 0
    out = torch.zeros_like(v)
    ctx.ssm_prompt(0, desc, _i32([0]), 1, _i32([0, tot]), tot, _i32([1]), q, k, v, g, out, torch.empty(size, dtype=torch.uint8, device="cuda"), size)
    S, o, _ = _recurrence(first.view(heads, dv, dk).double(), q, k, v, g, heads)
    z = lambda x: torch.nan_to_num(x, 0.0, 0.0, -math.inf if x is g else 0.0)
    mass = _recurrence(z(first).view(heads, dv, dk).double(), z(q), z(k), z(v), z(g), heads)[2]
    for a, b in ((0, 300), (300, 900), (900, 2900), (2900, 3300), (3300, tot)):
        _near(out[a:b], o[a:b], mass[a:b], f"rows {a} to {b}")
    _near_state(_states(ctx, 0, [0], m)[0].view(heads, dv, dk), S, -(-tot // 64), "state")
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("every", [2, 3, 7])
def test_many_resets_in_a_piece(every, dtype):
    import torch
    from paper_2605_22416_b200 import binding as B
    heads, dk, dv, tot = 3, 16, 64, 200
    dt, m = getattr(torch, dtype), _model(heads, dk, dv)
    ctx = _ctx(m, 2, [0])
    gen = torch.Generator("cuda").manual_seed(every)
    q, k = ((torch.randn(tot, 1, dk, device="cuda", generator=gen) * 0.3).to(dt) for _ in range(2))
    v = torch.randn(tot, heads, dv, device="cuda", generator=gen).to(dt)
    g = -torch.rand(tot, heads, device="cuda", generator=gen) * 0.5
    g[::every] = -math.inf
    out = torch.zeros_like(v)
    ctx.ssm_prompt(0, B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=dt), _i32([0]), 1, _i32([0, tot]), tot, None, q, k, v, g, out)
    S, o, mass = _recurrence(torch.zeros(heads, dv, dk, dtype=torch.float64, device="cuda"), q, k, v, g, heads)
    _near(out, o, mass, "rows")
    _near_state(_states(ctx, 0, [0], m)[0].view(heads, dv, dk), S, 4, "state")
    ctx.close()
