"""Waits inside the kernels that run out: the call is reported (AVMP_DEV_TIMEOUT), or its results are right; nothing outside its
outputs is written, and the calls behind it are as ever."""
from __future__ import annotations

import numpy as np
import pytest

from test_attn_ops import NONE, Cache, _i32
from test_ssm_ops import _ctx, _model


def test_the_limit_needs_a_context():
    from paper_2605_22416_b200 import binding as B
    assert B.lib.avmp_set_wait_limit(None, 5) == B.AVMP_EINVAL


def _attention(call, dtype):
    import torch
    from paper_2605_22416_b200 import binding as B
    held, dim = [900, 33, 260, 700], 64 if call == "prompt of few rows" else 128
    c = Cache(held, 4, dim, 16, dtype, seed=70)
    hq = 16 if call != "prompt of odd groups" else 12
    desc = B.attn_desc(q_heads=hq, dtype=c.dt, scale=0.1)
    ws, size = c.workspace(desc, 3)
    if call.startswith("prompt"):
        new = [5, 2, 3] if call == "prompt of few rows" else held[:3]
        tot, cu = sum(new), np.concatenate([[0], np.cumsum(new)])
    else:
        tot = 3
    q, _ = c.queries(tot, hq)
    out = torch.empty(tot + 1, hq, dim, dtype=c.dt, device="cuda")
    reqs = _i32([0, 1, 2])

    def run():
        out.fill_(7)
        if call.startswith("prompt"):
            c.ctx.attn_prompt(c.layer, desc, reqs, 3, _i32(cu), tot, q, out, None, ws, size)
        else:
            c.ctx.attn_decode(c.layer, desc, reqs, 3, 3 if call == "prefix" else NONE, q, out, None, ws, size)
        return [out[:tot].clone()], bool((out[tot:] == 7).all())

    return c.ctx, run


def _recurrence(call, dtype):
    import torch
    from paper_2605_22416_b200 import binding as B
    dt = getattr(torch, dtype)
    heads, dk, dv, lens = {"cut recurrence": (2, 128, 64, [2500, 40]), "recurrence": (40, 16, 64, [300, 64, 511]),
                           "long keys' recurrence": (40, 128, 64, [300, 64, 511])}[call]
    m, n, tot = _model(heads, dk, dv), len(lens), sum(lens)
    ctx = _ctx(m, 6, list(range(n)))
    gen = torch.Generator("cuda").manual_seed(1)
    q, k = ((torch.randn(tot, 1, dk, device="cuda", generator=gen) * 0.2).to(dt) for _ in range(2))
    v = torch.randn(tot, heads, dv, device="cuda", generator=gen).to(dt)
    g = -torch.rand(tot, heads, device="cuda", generator=gen) * 0.1
    desc = B.ssm_desc(heads=heads, groups=1, dk=dk, dv=dv, dtype=dt)
    size = ctx.ssm_workspace_bytes(desc, n, tot)
    ws = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")
    out, st = torch.empty(tot + 1, heads, dv, dtype=dt, device="cuda"), torch.empty(n, heads * dk * dv, device="cuda")
    cu = _i32(np.concatenate([[0], np.cumsum(lens)]))

    def run():
        out.fill_(7)
        ctx.ssm_prompt(0, desc, _i32(range(n)), n, cu, tot, None, q, k, v, g, out, ws, size)
        ctx.gather_ssm(0, _i32(range(n)), n, st, torch.empty(n, m.ssm_conv_elems, device="cuda"))
        return [out[:tot].clone(), st.clone()], bool((out[tot:] == 7).all())

    return ctx, run


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("call", ["prompt", "prompt of odd groups", "prompt of few rows", "decode", "prefix", "recurrence", "long keys' recurrence", "cut recurrence"])
def test_a_wait_that_runs_out_is_reported(call, dtype):
    import torch
    ctx, run = (_recurrence if call.endswith("recurrence") else _attention)(call, dtype)
    want, clean = run()
    assert clean and ctx.stats()["error_count"] == 0
    reported = 0
    for ns in [0, 0, 200, 500, 1000, 1500, 2000, 3000, 5000, 8000, 20000, 100000]:
        ctx.set_wait_limit(ns)
        got, clean = run()
        s = ctx.stats()
        assert clean, f"limit {ns}: rows behind the last are written"
        if s["error_count"]:
            assert s["error_code"] == 4
            reported += 1
            ctx.clear_error()
        else:
            assert all(torch.equal(a, b) for a, b in zip(got, want)), f"limit {ns}: wrong and not reported"
        # (the rows of short keys are asked for a piece ahead and may always be there)
        assert ns or s["error_count"] or call == "recurrence", "no wait ran out"
    ctx.set_wait_limit(10 ** 18)
    for _ in range(2):
        got, clean = run()
        assert clean and all(torch.equal(a, b) for a, b in zip(got, want)) and ctx.stats()["error_count"] == 0
    assert reported >= 2 or call == "recurrence"
    ctx.close()
