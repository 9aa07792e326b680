"""The linear recurrence on the SSM state blocks (avmp_ssm_prompt, avmp_ssm_step) against the recurrence itself in 64
bits, token by token.

Tolerances.  The state is summed in 32 bits from products of 16-bit inputs; e^(..) v is held as two 16-bit parts, which
leaves a relative error of at most (eps/2)^2 of the 16-bit type (2^-16 for bf16) per product; the exponentials add a few
2^-22 each and every piece of 64 tokens one more rounding.  Norm-wise that stays under 2^-16 plus 2^-18.  An output is
rounded once to 16 bits (eps/2), and two of its operands are (the decayed scores, the carried state): 3 * eps/2 of the
largest terms it is summed from, which norm-wise bounds the error by 3 * eps/2 times the norm of the sums of absolute
values; a factor of 2 covers that against the norm of the outputs, whose terms have random signs here.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import pytest

from paper_2605_22416_b200 import workloads as W


def _model(heads, dk, dv, layers=2, conv=100, elem=4):
    return SimpleNamespace(n_attn_layers=1, n_ssm_layers=layers, page_tokens=16, kv_heads=1, head_dim=64, kv_elem_bytes=2,
                           ssm_state_elems=heads * dk * dv, ssm_conv_elems=conv, ssm_elem_bytes=elem)


def _ctx(model, slots, live, seed=0):
    """A context whose slots `live` are admitted in a scrambled order, so that blocks are not in slot order."""
    from paper_2605_22416_b200 import binding as B
    u_ssm = -(-4 * (model.ssm_state_elems + model.ssm_conv_elems) // 16) * 16
    n = slots * model.n_ssm_layers + 3
    pool = int((n * u_ssm + (slots + 4) * 2 * 16 * 128) * 1.1) + 4096
    ctx = B.Context(model, pool, n * u_ssm / pool, 4, max_requests=slots, max_pages=4)
    order = np.random.default_rng(seed).permutation(np.asarray(live))
    st = np.zeros(len(order), np.uint32)
    ctx.step_host(W.make_ops(W.OP_ADMIT, order, 5), len(order), st)
    assert (st == 0).all()
    return ctx


def _i32(x):
    import torch
    return torch.tensor(np.asarray(x, np.int64).astype(np.uint32).view(np.int32), device="cuda")


def _rows(shape, dtype, gen, scale, pad=0):
    """Rows of `shape` inside a wider buffer (pad elements behind each row): (view, row stride in bytes)."""
    import torch
    n, width = shape[0], int(np.prod(shape[1:]))
    buf = (torch.randn(n, width + pad, device="cuda", generator=gen) * scale).to(dtype)
    return buf[:, :width].view(n, *shape[1:]) if pad == 0 else buf[:, :width].unflatten(1, shape[1:]), (width + pad) * buf.element_size()


def _states(ctx, layer, reqs, model):
    import torch
    n = len(reqs)
    st = torch.empty(n, model.ssm_state_elems, dtype=torch.float32, device="cuda")
    cv = torch.empty(n, model.ssm_conv_elems, dtype=torch.float32, device="cuda")
    ctx.gather_ssm(layer, _i32(reqs), n, st, cv)
    return st, cv


def _recurrence(S, q, k, v, g, rep):
    """64 bits: S [heads, dv, dk] (changed), rows of one request."""
    import torch
    out = torch.zeros(v.shape, dtype=torch.float64, device=v.device)
    for t in range(v.shape[0]):
        w = g[t].double().exp()[:, None, None]
        S = torch.where(w == 0, torch.zeros_like(S), S * w) + v[t].double()[:, :, None] * k[t].double().repeat_interleave(rep, 0)[:, None, :]
        out[t] = (S * q[t].double().repeat_interleave(rep, 0)[:, None, :]).sum(-1)
    return S, out


def _check(got, want, tol, what):
    import torch
    assert torch.isfinite(got).all(), what
    err = float((got.double() - want).norm() / want.norm().clamp(min=1e-300))
    assert err <= tol, f"{what}: relative error {err:.3g} over {tol:.3g}"


def _out_tol(dtype):
    import torch
    return 2 * 3 * torch.finfo(dtype).eps / 2


STATE_TOL = 2.0 ** -16 + 2.0 ** -18


def _fill_state(ctx, layer, reqs, model, gen, scale=1.0):
    import torch
    n = len(reqs)
    st = torch.randn(n, model.ssm_state_elems, device="cuda", generator=gen) * scale
    cv = torch.randn(n, model.ssm_conv_elems, device="cuda", generator=gen)
    ctx.scatter_ssm(layer, _i32(reqs), n, st, cv)
    return st, cv


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("heads,groups,dk,dv", [(1, 1, 16, 32), (3, 1, 16, 64), (8, 2, 32, 96), (6, 3, 64, 64), (4, 4, 128, 32), (2, 1, 128, 128)])
def test_single_tokens(dtype, heads, groups, dk, dv):
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = getattr(torch, dtype)
    m = _model(heads, dk, dv)
    reqs = [7, 2, 11, 0, 5]
    ctx = _ctx(m, 12, reqs + [3])
    gen = torch.Generator("cuda").manual_seed(heads * 1000 + dk)
    n, layer = len(reqs), 1
    first, conv = _fill_state(ctx, layer, reqs, m, gen)
    other, _ = _fill_state(ctx, 0, reqs, m, gen)
    bystander, _ = _fill_state(ctx, layer, [3], m, gen)
    q, qs = _rows((n, groups, dk), dt, gen, dk ** -0.5, pad=8)
    k, ks = _rows((n, groups, dk), dt, gen, 1.0, pad=16)
    v, vs = _rows((n, heads, dv), dt, gen, 0.5, pad=24)
    g = (-torch.rand(n, heads + 1, device="cuda", generator=gen))[:, :heads]
    g[1, 0] = -math.inf                                   # clears that head's state
    out = torch.full((n, heads * dv + 8), 7.0, dtype=dt, device="cuda")
    desc = B.ssm_desc(heads=heads, groups=groups, dk=dk, dv=dv, dtype=dt, q_stride_bytes=qs, k_stride_bytes=ks,
                      v_stride_bytes=vs, decay_stride_bytes=(heads + 1) * 4, out_stride_bytes=(heads * dv + 8) * 2)
    ctx.ssm_step(layer, desc, _i32(reqs), n, q, k, v, g, out)
    st, cv = _states(ctx, layer, reqs, m)
    for i in range(n):
        S, o = _recurrence(first[i].view(heads, dv, dk).double(), q[i:i + 1], k[i:i + 1], v[i:i + 1], g[i:i + 1], heads // groups)
        _check(st[i].view(heads, dv, dk), S, 2.0 ** -21, f"state {i}")
        _check(out[i, :heads * dv].view(1, heads, dv), o, torch.finfo(dt).eps / 2, f"out {i}")
    assert (out[:, heads * dv:] == 7).all() and torch.equal(cv, conv)
    assert torch.equal(_states(ctx, 0, reqs, m)[0], other) and torch.equal(_states(ctx, layer, [3], m)[0], bystander)
    assert ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,heads,groups,dk,dv", [(120, 128, 8, 16, 128), (67, 37, 1, 128, 96), (330, 20, 4, 64, 64)])
def test_single_tokens_of_large_states(dtype, n, heads, groups, dk, dv):
    """Batches of many CTAs per request, with ends of blocks inside a CTA's part and skipped entries in the list; twice."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = getattr(torch, dtype)
    m = _model(heads, dk, dv, layers=1, conv=20)
    slots = n + 5
    ctx = _ctx(m, slots, list(range(n)))
    gen = torch.Generator("cuda").manual_seed(n)
    order = np.random.default_rng(n).permutation(n)
    reqs = list(order[: n - 3]) + [order[0], n + 2, 0xFFFFFFFF]           # named before, empty, out of range
    first, conv = _fill_state(ctx, 0, order, m, gen)
    q, k = ((torch.randn(n, groups, dk, device="cuda", generator=gen) * 0.2).to(dt) for _ in range(2))
    v = (torch.randn(n, heads, dv, device="cuda", generator=gen)).to(dt)
    g = -torch.rand(n, heads, device="cuda", generator=gen)
    g[5, 0] = -math.inf
    out = torch.full((n, heads, dv), 7.0, dtype=dt, device="cuda")
    desc = B.ssm_desc(heads=heads, groups=groups, dk=dk, dv=dv, dtype=dt)
    for step in range(2):
        ctx.ssm_step(0, desc, _i32(reqs), n, q, k, v, g, out)
        assert ctx.stats()["error_count"] == 3 * (step + 1)
    st, cv = _states(ctx, 0, order, m)
    S = first.view(n, heads, dv, dk)[: n - 3].double()
    rep = heads // groups
    kk, qq = (x[: n - 3].double().repeat_interleave(rep, 1)[:, :, None, :] for x in (k, q))
    w = g[: n - 3].double().exp()[:, :, None, None]
    for _ in range(2):
        S = torch.where(w == 0, torch.zeros_like(S), S * w) + v[: n - 3].double()[..., None] * kk
    _check(st.view(n, heads, dv, dk)[: n - 3], S, 2.0 ** -20, "states")
    _check(out[: n - 3], (S * qq).sum(-1), torch.finfo(dt).eps / 2, "out")
    assert torch.equal(st[n - 3:], first[n - 3:]) and (out[n - 3:] == 7).all() and torch.equal(cv, conv)
    ctx.close()


PROMPTS = [
    # heads, groups, dk, dv, lengths, resume
    (1, 1, 16, 32, [1], [0]),
    (3, 1, 16, 64, [0, 1, 63, 64, 65, 200], [0, 1, 0, 1, 1, 0]),
    (4, 2, 32, 64, [257, 2, 0, 128], [1, 1, 1, 0]),
    (2, 2, 64, 96, [130, 64, 7], [0, 1, 0]),
    (4, 1, 64, 128, [191, 1], [1, 1]),
    (2, 1, 128, 64, [65, 300, 12], [1, 0, 1]),
    (2, 2, 128, 32, [129], [1]),
    (40, 8, 16, 64, [1000, 17, 513], [1, 1, 0]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(PROMPTS)))
def test_prompts(dtype, case):
    import torch
    from paper_2605_22416_b200 import binding as B
    heads, groups, dk, dv, lens, resume = PROMPTS[case]
    dt = getattr(torch, dtype)
    m = _model(heads, dk, dv)
    n, layer = len(lens), 1
    reqs = [(5 * i + 3) % 13 for i in range(n)]
    ctx = _ctx(m, 13, reqs)
    gen = torch.Generator("cuda").manual_seed(case)
    first, conv = _fill_state(ctx, layer, reqs, m, gen)
    for i in range(n):
        if not resume[i]:        # what a fresh block holds is not read
            ctx.scatter_ssm(layer, _i32([reqs[i]]), 1, torch.full((1, m.ssm_state_elems), math.nan, device="cuda"), conv[i:i + 1].clone())
    tot = sum(lens)
    cu = np.concatenate([[0], np.cumsum(lens)])
    q, qs = _rows((tot + 2, groups, dk), dt, gen, dk ** -0.5, pad=8)
    k, ks = _rows((tot + 2, groups, dk), dt, gen, 1.0)
    v, vs = _rows((tot + 2, heads, dv), dt, gen, 0.5, pad=16)
    g = -torch.rand(tot + 2, heads, device="cuda", generator=gen) ** 4
    g[:, 0] *= 20
    if tot > 70:
        g[cu[-1] - 40, heads - 1] = -math.inf
    out = torch.full((tot + 2, heads, dv), 7.0, dtype=dt, device="cuda")
    desc = B.ssm_desc(heads=heads, groups=groups, dk=dk, dv=dv, dtype=dt, q_stride_bytes=qs, k_stride_bytes=ks, v_stride_bytes=vs)
    ctx.ssm_prompt(layer, desc, _i32(reqs), n, _i32(cu), tot + 2, _i32(resume), q, k, v, g, out)
    st, cv = _states(ctx, layer, reqs, m)
    for i in range(n):
        S0 = first[i].view(heads, dv, dk).double() * resume[i]
        a, b = cu[i], cu[i + 1]
        S, o = _recurrence(S0, q[a:b], k[a:b], v[a:b], g[a:b], heads // groups)
        if lens[i]:
            _check(st[i].view(heads, dv, dk), S, STATE_TOL, f"state {i}")
            _check(out[a:b], o, _out_tol(dt), f"out {i}")
        else:
            assert torch.equal(st[i].view(heads, dv, dk), S.float())
    assert (out[tot:] == 7).all() and torch.equal(cv, conv)       # rows behind the last prompt, windows
    assert ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,heads,dk,dv,lens,resume", [("bfloat16", 1, 16, 64, [9001], [1]), ("float16", 2, 64, 32, [20, 0, 6000], [1, 1, 0]),
                                                           ("bfloat16", 3, 128, 64, [4097, 65], [0, 1]), ("bfloat16", 1, 32, 32, [2048], [0])])
def test_long_prompts_of_few_heads(dtype, heads, dk, dv, lens, resume):
    """Prompts that are cut into runs over the SMs: same state and outputs; short and empty requests beside them; a reset inside."""
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = getattr(torch, dtype)
    m = _model(heads, dk, dv)
    n, tot = len(lens), sum(lens)
    ctx = _ctx(m, 6, list(range(n)))
    gen = torch.Generator("cuda").manual_seed(dk)
    first, conv = _fill_state(ctx, 1, list(range(n)), m, gen)
    q, k = ((torch.randn(tot, 1, dk, device="cuda", generator=gen) * 0.2).to(dt) for _ in range(2))
    v = torch.randn(tot, heads, dv, device="cuda", generator=gen).to(dt)
    g = -torch.rand(tot, heads, device="cuda", generator=gen) ** 6 * 0.2
    g[tot // 2, 0] = -math.inf
    desc = B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=dt)
    cu = np.concatenate([[0], np.cumsum(lens)])
    size = ctx.ssm_workspace_bytes(desc, n, tot)
    assert size > 0
    with pytest.raises(B.AvmpError, match="invalid argument"):
        ctx.ssm_prompt(1, desc, _i32(range(n)), n, _i32(cu), tot, _i32(resume), q, k, v, g, v)
    ws = torch.full((size + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.AvmpError, match="workspace too small"):
        ctx.ssm_prompt(1, desc, _i32(range(n)), n, _i32(cu), tot, _i32(resume), q, k, v, g, v, ws, size - 16)
    for rep in range(2):
        ctx.scatter_ssm(1, _i32(range(n)), n, first, conv)
        out = torch.zeros_like(v)
        ctx.ssm_prompt(1, desc, _i32(range(n)), n, _i32(cu), tot, _i32(resume), q, k, v, g, out, ws, size)
    st, cv = _states(ctx, 1, list(range(n)), m)
    for i in range(n):
        a, b = cu[i], cu[i + 1]
        S, o = _recurrence(first[i].view(heads, dv, dk).double() * resume[i], q[a:b], k[a:b], v[a:b], g[a:b], heads)
        if lens[i]:
            _check(st[i].view(heads, dv, dk), S, STATE_TOL, f"state {i}")
            _check(out[a:b], o, _out_tol(dt), f"out {i}")
        else:
            assert torch.equal(st[i].view(heads, dv, dk), S.float())
    assert (ws[size:] == 0xFF).all() and torch.equal(cv, conv) and ctx.stats()["error_count"] == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [2.0 ** -12, 2.0 ** 9])
def test_half_precision_inputs_of_extreme_size(scale):
    """fp16 rows near the ends of their range: scores and states pass 65504 and fall below 2^-14."""
    import torch
    from paper_2605_22416_b200 import binding as B
    heads, dk, dv, tot = 2, 64, 64, 150
    m = _model(heads, dk, dv)
    ctx = _ctx(m, 2, [1])
    gen = torch.Generator("cuda").manual_seed(3)
    q, k = ((torch.randn(tot, 1, dk, device="cuda", generator=gen) * scale).half() for _ in range(2))
    v = (torch.randn(tot, heads, dv, device="cuda", generator=gen) * 2.0 ** -4).half()
    g = -torch.rand(tot, heads, device="cuda", generator=gen) * 0.1
    out = torch.zeros(tot, heads, dv, dtype=torch.float16, device="cuda")
    S, o = _recurrence(torch.zeros(heads, dv, dk, dtype=torch.float64, device="cuda"), q, k, v, g, heads)
    if scale < 1:
        v = (v.float() * 2.0 ** 15).half()                    # outputs in the range of fp16 again
        S, o = S * 2.0 ** 15, o * 2.0 ** 15
    else:
        v = (v.float() * 2.0 ** -9).half()
        S, o = _recurrence(torch.zeros_like(S), q, k, v, g, heads)
    assert float(o.abs().max()) < 65504
    ctx.ssm_prompt(0, B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=torch.float16), _i32([1]), 1, _i32([0, tot]), tot,
                   None, q, k, v, g, out)
    _check(_states(ctx, 0, [1], m)[0].view(heads, dv, dk), S, STATE_TOL, "state")
    _check(out, o, _out_tol(torch.float16), "out")
    ctx.close()


@pytest.mark.gpu
def test_prompt_then_tokens_equals_one_prompt():
    """A prompt in two chunks and a few single tokens behind it leave the state and the outputs of one long prompt."""
    import torch
    from paper_2605_22416_b200 import binding as B
    heads, groups, dk, dv, tot = 4, 2, 16, 64, 203
    m = _model(heads, dk, dv)
    ctx = _ctx(m, 4, [0, 1, 2])
    gen = torch.Generator("cuda").manual_seed(9)
    dt = torch.bfloat16
    q, k = ((torch.randn(tot, groups, dk, device="cuda", generator=gen) * 0.5).to(dt) for _ in range(2))
    v = torch.randn(tot, heads, dv, device="cuda", generator=gen).to(dt)
    g = -torch.rand(tot, heads, device="cuda", generator=gen)
    desc = B.ssm_desc(heads=heads, groups=groups, dk=dk, dv=dv, dtype=dt)
    whole, parts = torch.zeros_like(v), torch.zeros_like(v)
    ctx.ssm_prompt(0, desc, _i32([2]), 1, _i32([0, tot]), tot, None, q, k, v, g, whole)
    at = 0
    for end in (90, 200):
        n = end - at
        ctx.ssm_prompt(0, desc, _i32([0]), 1, _i32([0, n]), n, _i32([1 if at else 0]), q[at:end], k[at:end], v[at:end], g[at:end], parts[at:end])
        at = end
    for t in range(at, tot):
        ctx.ssm_step(0, desc, _i32([0]), 1, q[t:t + 1], k[t:t + 1], v[t:t + 1], g[t:t + 1], parts[t:t + 1])
    S, o = _recurrence(torch.zeros(heads, dv, dk, dtype=torch.float64, device="cuda"), q, k, v, g, heads // groups)
    for r, out in ((2, whole), (0, parts)):
        _check(_states(ctx, 0, [r], m)[0].view(heads, dv, dk), S, STATE_TOL, f"state {r}")
        _check(out, o, _out_tol(dt), f"out {r}")
    ctx.close()


@pytest.mark.gpu
def test_bad_items_are_skipped():
    import torch
    from paper_2605_22416_b200 import binding as B
    heads, dk, dv = 2, 16, 32
    m = _model(heads, dk, dv)
    ctx = _ctx(m, 8, [0, 1, 2, 3])
    st = np.zeros(1, np.uint32)
    ctx.step_host(W.make_ops(W.OP_FINISH, [3], 0, W.FLAG_KEEP_KV), 1, st)      # parked: holds no state blocks
    gen = torch.Generator("cuda").manual_seed(1)
    before, _ = _fill_state(ctx, 0, [0, 1, 2], m, gen)
    desc = B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=torch.bfloat16)

    def rows(n):
        return ((torch.randn(n, 1, dk, device="cuda", generator=gen)).bfloat16(), torch.randn(n, 1, dk, device="cuda", generator=gen).bfloat16(),
                torch.randn(n, heads, dv, device="cuda", generator=gen).bfloat16(), -torch.rand(n, heads, device="cuda", generator=gen))

    reqs = [1, 3, 1, 6, 0xFFFFFFFF]              # fine, parked, named before, empty, out of range
    q, k, v, g = rows(5)
    out = torch.full((5, heads, dv), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.ssm_step(0, desc, _i32(reqs), 5, q, k, v, g, out)
    s = ctx.stats()
    assert s["error_count"] == 4 and s["error_code"] == 2
    assert (out[1:] == 7).all() and not (out[0] == 7).all()
    now = _states(ctx, 0, [0, 1, 2], m)[0]
    assert torch.equal(now[[0, 2]], before[[0, 2]]) and not torch.equal(now[1], before[1])
    ctx.clear_error()
    # prompts: repeated slot, decreasing offsets, offsets past the buffers
    q, k, v, g = rows(20)
    out = torch.full((20, heads, dv), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.ssm_prompt(0, desc, _i32([0, 0, 1, 2]), 4, _i32([0, 4, 9, 8, 21]), 20, None, q, k, v, g, out)
    assert ctx.stats()["error_count"] == 3
    assert (out[4:] == 7).all() and not (out[:4] == 7).all()
    after = _states(ctx, 0, [0, 1, 2], m)[0]
    assert torch.equal(after[1:], now[1:]) and not torch.equal(after[0], now[0])
    ctx.close()


@pytest.mark.gpu
def test_graph_replay_other_stream_and_empty_lists():
    import torch
    from paper_2605_22416_b200 import binding as B
    heads, dk, dv, tot = 2, 32, 64, 100
    m = _model(heads, dk, dv)
    ctx = _ctx(m, 4, [0, 1])
    gen = torch.Generator("cuda").manual_seed(4)
    dt = torch.bfloat16
    q, k = ((torch.randn(tot, 1, dk, device="cuda", generator=gen) * 0.3).to(dt) for _ in range(2))
    v = torch.randn(tot, heads, dv, device="cuda", generator=gen).to(dt)
    g = -torch.rand(tot, heads, device="cuda", generator=gen)
    desc = B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=dt)
    ctx.ssm_step(0, desc, 0, 0, 0, 0, 0, 0, 0)
    ctx.ssm_prompt(0, desc, 0, 0, 0, 0, None, 0, 0, 0, 0, 0)
    reqs, cu, last = _i32([1, 0]), _i32([0, 70, 100]), slice(98, 100)
    out, tail = torch.zeros_like(v), torch.zeros(2, heads, dv, dtype=dt, device="cuda")

    def both():
        ctx.ssm_prompt(1, desc, reqs, 2, cu, tot, None, q, k, v, g, out)
        ctx.ssm_step(1, desc, reqs, 2, q[last], k[last], v[last], g[last], tail)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    want, want_tail, want_state = out.clone(), tail.clone(), _states(ctx, 1, [0, 1], m)[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        out.zero_(); tail.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(tail, want_tail) and torch.equal(_states(ctx, 1, [0, 1], m)[0], want_state)
    ctx.close()


@pytest.mark.gpu
def test_no_tokens_at_all():
    """A list whose requests bring no rows: states are cleared, or kept where they are resumed; the row buffers may be absent."""
    import torch
    from paper_2605_22416_b200 import binding as B
    heads, dk, dv = 2, 64, 64
    m = _model(heads, dk, dv)
    ctx = _ctx(m, 4, [0, 1, 2])
    gen = torch.Generator("cuda").manual_seed(4)
    before, _ = _fill_state(ctx, 1, [0, 1, 2], m, gen)
    desc = B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=torch.bfloat16)
    ctx.ssm_prompt(1, desc, _i32([2, 0]), 2, _i32([0, 0, 0]), 0, _i32([0, 1]), None, None, None, None, None)
    after, _ = _states(ctx, 1, [0, 1, 2], m)
    assert torch.equal(after[:2], before[:2]) and (after[2] == 0).all() and ctx.stats()["error_count"] == 0
    ctx.close()


def test_refusals_on_the_host():
    """Arguments are checked before anything is launched (a made-up context on host memory: never dereferenced)."""
    import ctypes
    from paper_2605_22416_b200 import binding as B
    with pytest.raises(B.AvmpError):
        import torch
        B.ssm_desc(heads=1, groups=1, dk=16, dv=32, dtype=torch.float32)
    assert B.lib.avmp_ssm_step(None, 0, ctypes.byref(B.avmp_ssm_desc()), None, 1, None, None, None, None, None, None) == B.AVMP_EINVAL
    assert B.lib.avmp_ssm_prompt(None, 0, ctypes.byref(B.avmp_ssm_desc()), None, 1, None, 0, None, None, None, None, None, None,
                                 None, 0, None) == B.AVMP_EINVAL


@pytest.mark.gpu
def test_refusals():
    import torch
    from paper_2605_22416_b200 import binding as B
    heads, dk, dv = 2, 16, 32
    m = _model(heads, dk, dv)
    ctx = _ctx(m, 4, [0])
    x = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    f = torch.zeros(64, device="cuda")
    ok = dict(heads=heads, groups=1, dk=dk, dv=dv, dtype=torch.bfloat16)
    reqs, cu = _i32([0]), _i32([0, 1])

    def step(layer=0, n=1, q=x, g=f, reqs=reqs, **kw):
        ctx.ssm_step(layer, B.ssm_desc(**{**ok, **kw}), reqs, n, q, x, x, g, x)

    def prompt(layer=0, n=1, q=x, cu=cu, total=1, **kw):
        ctx.ssm_prompt(layer, B.ssm_desc(**{**ok, **kw}), reqs, n, cu, total, None, q, x, x, f, x)

    bad = [dict(layer=2), dict(n=5), dict(heads=4), dict(groups=0), dict(dk=8, dv=64), dict(dk=32, dv=16), dict(heads=1, dv=64, groups=2),
           dict(q_stride_bytes=24), dict(v_stride_bytes=64), dict(q=x.data_ptr() + 2), dict(q=None), dict(decay_stride_bytes=6)]
    for kw in bad:
        with pytest.raises(B.AvmpError, match="invalid argument"):
            step(**kw)
        if "decay_stride_bytes" not in kw:
            with pytest.raises(B.AvmpError, match="invalid argument"):
                prompt(**kw)
    for kw in (dict(g=f.data_ptr() + 2), dict(reqs=None)):
        with pytest.raises(B.AvmpError, match="invalid argument"):
            step(**kw)
    with pytest.raises(B.AvmpError, match="invalid argument"):
        prompt(cu=None)
    assert ctx.stats()["error_count"] == 0
    ctx.close()
    two = _ctx(_model(heads, dk * 2, dv, elem=2), 4, [0])          # a 2-byte state store
    with pytest.raises(B.AvmpError, match="invalid argument"):
        two.ssm_step(0, B.ssm_desc(heads=heads, groups=1, dk=dk * 2, dv=dv, dtype=torch.bfloat16), reqs, 1, x, x, x, f, x)
    two.close()
