"""Cases for the operators of a hybrid layer around its caches: the short causal convolution on a state block's window,
the selective scan on its state, norms and rotation of query and key heads with the write into the KV pages, and attention
with a sliding window and sinks over the paged chains; each for prompts and for single tokens.

`own` false: the plain form, elementary torch operations in 32 bits.  `own` true: the library's entry points.
Both work on the same arena: KV pages and state blocks lie at random physical slots and are reached through a table.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
LENGTHS = {"len_seed": 1, "long_share": 0.0, "long_lo": 1, "long_hi": 1}


# ---------------------------------------------------------------- cases
def _state(op, **kw):
    return {"op": op, "dtype": "bf16", "channels": 2048, "width": 4, "states": 16, "groups": 1, "layers": 2, "layer": 1, "resume": 0,
            "bias": True, **LENGTHS, **kw}


def _attn(op, **kw):
    return {"op": op, "dtype": "bf16", "page_tokens": 16, "kv_heads": 8, "q_heads": 32, "head_dim": 128, "layers": 2, "layer": 1,
            **LENGTHS, **kw}


def listed():
    return [
        # a long document and short prompts, half of them continued from a kept window
        _state("conv_prompt", name="conv_prompt_long", n=5, lo=1, hi=2000, channels=8192, long_share=0.2, long_lo=65521, long_hi=65521, resume=1,
               len_seed=8),
        # decode step of a full `pr1` batch: latency counts
        _state("conv_step", name="conv_step_pr1", n=32),
        # the state layers of the `pr1` admission step: 32 short prompts of very different lengths
        _state("scan_prompt", name="scan_prompt_pr1", n=32, lo=32, hi=512),
        # a long document beside short prompts, half of them continued from a kept state
        _state("scan_prompt", name="scan_prompt_long", n=5, lo=1, hi=2000, channels=8192, dtype="f16", long_share=0.2, long_lo=32749,
               long_hi=32749, resume=1, len_seed=9),
        # decode step of `pr1`, and of `scale` (one megabyte of state for each request)
        _state("scan_step", name="scan_step_pr1", n=32),
        _state("scan_step", name="scan_step_scale", n=1023, channels=16384, layers=1, layer=0),
        # sessions that come back: each appends a turn of 256 to 2048 tokens to a chain that was kept between turns
        _attn("rows_prompt", name="rows_prompt_sessions", n=12, lo=256, hi=2048, past_lo=1, past_hi=8192, q_heads=64, rotary=128,
              neighbours=False, norm=True, len_seed=2),
        # decode step of the `scale` workload's 1024 running requests
        _attn("rows_step", name="rows_step_scale", n=1024, lo=40, hi=600, rotary=64, neighbours=True, norm=True, dtype="f16", len_seed=4),
        # turns of sessions again, seen through a window
        _attn("prompt", name="window_prompt_sessions", n=12, lo=256, hi=2048, past_lo=1, past_hi=8192, window=1024, sinks=4, dtype="f16",
              len_seed=2),
        # one prompt of the `mixed_long` kind beside three ordinary ones, one of them a single token
        _attn("prompt", name="window_prompt_long", n=4, lo=1, hi=900, past_lo=0, past_hi=0, window=4096, sinks=16, long_share=0.25,
              long_lo=32749, long_hi=32749, len_seed=3),
        # decode step of a full `pr1` batch, most chains shorter than the window
        _attn("decode", name="window_decode_pr1", n=32, lo=48, hi=640, window=512, sinks=4),
        # decode step of `mixed_long`: a fifth of the batch holds 16 to 64 thousand tokens, of which the window shows a part
        _attn("decode", name="window_decode_mixed_long", n=128, lo=100, hi=8000, window=4096, sinks=4, long_share=0.2, long_lo=16384,
              long_hi=65536, layers=1, layer=0, len_seed=5),
    ]


def _logu(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["conv_prompt", "conv_step", "scan_prompt", "scan_step", "rows_prompt", "rows_step", "prompt", "decode"])
    seed, dtype = rng.randrange(1 << 30), rng.choice(["bf16", "f16"])
    if op.startswith(("conv", "scan")):
        groups = rng.choice([1, 1, 2, 4])
        channels = groups * 8 * _logu(rng, 8, 2048 // groups)
        states = rng.choice([8, 16, 16, 32, 64])
        kw = dict(channels=channels, groups=groups, states=states, width=rng.choice([2, 3, 4]), dtype=dtype, bias=rng.random() < 0.7,
                  resume=rng.randint(0, 1), len_seed=seed)
        # within the largest listed case's elements
        if op == "conv_step":
            return _state(op, n=_logu(rng, 1, min(1023, 16_000_000 // channels, (1 << 28) // (channels * states))), **kw)
        if op == "scan_step":
            return _state(op, n=_logu(rng, 1, min(1023, (1 << 28) // (channels * states))), **kw)
        n = _logu(rng, 1, 40)
        each = channels * (states if op == "scan_prompt" else 8)
        most = max(2, min(32768, 4_000_000_000 // (n * each)))
        lo = _logu(rng, 1, most)
        return _state(op, n=n, lo=lo, hi=_logu(rng, lo, most), **kw)
    kv_heads, head_dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    kw = dict(kv_heads=kv_heads, q_heads=kv_heads * rng.choice([1, 2, 3, 4, 8, 16]), head_dim=head_dim, dtype=dtype,
              page_tokens=rng.choice([16, 32, 64]), layers=2, layer=rng.randint(0, 1), len_seed=seed)
    if op.startswith("rows"):
        kw.update(rotary=rng.choice([0, head_dim // 4, head_dim // 2, head_dim]), neighbours=rng.random() < 0.5, norm=rng.random() < 0.7)
    else:
        kw.update(window=_logu(rng, 64, 8192), sinks=rng.choice([0, 1, 4, 16, 130]))
    if op == "rows_step":
        return _attn(op, n=_logu(rng, 1, 1024), lo=1, hi=_logu(rng, 1, 600), **kw)
    if op == "rows_prompt":
        n = _logu(rng, 1, 40)
        most = max(2, min(16384, 200_000_000 // (n * (kw["q_heads"] + 2 * kv_heads) * head_dim)))
        lo = _logu(rng, 1, most)
        return _attn(op, n=n, lo=lo, hi=_logu(rng, lo, most), past_lo=0, past_hi=rng.choice([0, 1]) * _logu(rng, 1, 8192), **kw)
    if op == "prompt":
        n = _logu(rng, 1, 40)
        most = max(2, min(16384, int(1e11 / (n * kw["q_heads"] * head_dim * min(kw["window"], 4096)))))
        lo = _logu(rng, 1, most)
        return _attn(op, n=n, lo=lo, hi=_logu(rng, lo, most), past_lo=0, past_hi=rng.choice([0, 1]) * _logu(rng, 1, 16384), **kw)
    n = _logu(rng, 1, 1024)
    most = max(16, min(65536, 800_000_000 // (n * kv_heads * head_dim)))
    lo = _logu(rng, 1, most)
    return _attn(op, n=n, lo=lo, hi=_logu(rng, lo, most), **kw)


def _lengths(case, lo, hi):
    """The case's own ragged lengths, spread over the logarithm; a share of them (at least one) from the long range."""
    r = random.Random(case["len_seed"] * 7919)
    v = [_logu(r, lo, hi) for _ in range(case["n"])]
    if case["long_share"] > 0:
        for i in r.sample(range(case["n"]), max(1, round(case["long_share"] * case["n"]))):
            v[i] = _logu(r, case["long_lo"], case["long_hi"])
    return v


def _plan(case):
    """(new tokens, tokens held) of each request."""
    op = case["op"]
    if op in ("conv_prompt", "scan_prompt"):
        return _lengths(case, case["lo"], case["hi"]), None
    if op in ("conv_step", "scan_step"):
        return [1] * case["n"], None
    if op in ("rows_prompt", "prompt"):
        new = _lengths(case, case["lo"], case["hi"])
        r = random.Random(case["len_seed"] + 17)
        return new, [a + r.randint(case["past_lo"], case["past_hi"]) for a in new]
    return [1] * case["n"], _lengths(case, case["lo"], case["hi"])


def work(case):
    new, held = _plan(case)
    tokens, op = sum(new), case["op"]
    if held is None:
        d, ns, w, n = case["channels"], case["states"], case["width"], case["n"]
        reads = n if op.endswith("step") else case["resume"] * (n // 2)
        if op.startswith("conv"):
            return {"bytes": 4 * tokens * d + 4 * d * (w - 1) * (n + reads) + 4 * d * (w + 1), "flops": 2 * tokens * d * w}
        # rows: u, step, gate and output of each channel, B and C; states; the decays, once
        return {"bytes": tokens * (2 * 4 * d + 4 * case["groups"] * ns) + 4 * d * ns * (n + reads) + 4 * d * ns, "flops": 7 * tokens * d * ns}
    hq, hk, dim = case["q_heads"], case["kv_heads"], case["head_dim"]
    if op.startswith("rows"):
        return {"bytes": 2 * 2 * tokens * (hq + 2 * hk) * dim, "flops": 8 * tokens * (hq + hk) * dim}
    w, s = case["window"], case["sinks"]

    def seen(p):      # keys that the rows at positions 0 .. p - 1 see, in all
        full = min(p, w)
        total = full * (full + 1) // 2 + (p - full) * w
        far = max(0, p - w)
        first = min(far, s)
        return total + first * (first + 1) // 2 + (far - first) * s

    pairs = sum(seen(b) - seen(b - a) for a, b in zip(new, held))
    keys = sum(min(b, a + w - 1) + min(s, max(0, b - (a + w - 1))) for a, b in zip(new, held))
    return {"bytes": 2 * 2 * hk * dim * keys + 2 * 2 * tokens * hq * dim + 4 * tokens * hq, "flops": 4 * hq * dim * pairs}


# ---------------------------------------------------------------- inputs
def _arena(case, n_kv, n_ssm):
    """Arena of n_kv pages and n_ssm blocks: pages grow from its base, block j ends j units before its end."""
    m = SimpleNamespace(n_attn_layers=1, n_ssm_layers=1, page_tokens=case.get("page_tokens", 16), kv_heads=case.get("kv_heads", 8),
                        head_dim=case.get("head_dim", 128), kv_elem_bytes=2, ssm_state_elems=8192 * 16, ssm_conv_elems=8192 * 3,
                        ssm_elem_bytes=4)
    if "channels" in case:
        m.n_ssm_layers = case["layers"]
        m.ssm_state_elems, m.ssm_conv_elems = case["channels"] * case["states"], case["channels"] * (case["width"] - 1)
    else:
        m.n_attn_layers = case["layers"]
    u_kv = m.n_attn_layers * 2 * m.page_tokens * m.kv_heads * m.head_dim * 2
    u_ssm = -(-4 * (m.ssm_state_elems + m.ssm_conv_elems) // 16) * 16
    pool = -(-(n_kv * u_kv + n_ssm * u_ssm) // 128) * 128
    return SimpleNamespace(model=m, u_kv=u_kv, u_ssm=u_ssm, pool=pool, n_kv=n_kv, n_ssm=n_ssm,
                           arena=torch.empty(pool, dtype=torch.uint8, device="cuda"))


def _handle(a, held, chains, blocks):
    """What a user of the library keeps beside the arena: a context whose tables hold these chains and blocks."""
    import numpy as np
    from paper_2605_22416_b200 import binding as B
    n = len(held)
    max_pages = max(len(c) for c in chains)
    ctx = B.Context(a.model, a.pool, 0.5, 16, max_requests=n, max_pages=max_pages, arena=a.arena, migration_enabled=False)
    t = {}
    for p, (nm, cap, used) in enumerate((("kv", a.n_kv, [s for c in chains for s in c]), ("ssm", a.n_ssm, [s for b in blocks for s in b]))):
        v, used = int(ctx.layout.vid_space[p]), np.asarray(used, np.int64)
        vt, ow = np.full(v, 0xFFFFFFFF, np.uint32), np.full(v, 0xFFFFFFFF, np.uint32)
        vt[: len(used)], ow[used] = used, np.arange(len(used))      # ids in order of use, slots anywhere
        t[f"slot_stack_{nm}"] = np.setdiff1d(np.arange(cap), used).astype(np.uint32)
        t[f"vid_stack_{nm}"] = np.arange(len(used), v).astype(np.uint32)
        t[f"vt_{nm}"], t[f"ow_{nm}"] = vt, ow
    t["req_state"] = np.full(n, 1 if blocks else 2, np.uint32)
    t["req_len"], t["req_npages"] = np.array(held, np.uint32), np.array([len(c) for c in chains], np.uint32)
    chain, at = np.zeros((n, max_pages), np.uint32), 0
    for i, c in enumerate(chains):
        chain[i, : len(c)] = np.arange(at, at + len(c))
        at += len(c)
    t["req_chain"] = chain.reshape(-1)
    ssm = np.full((n, a.model.n_ssm_layers), 0xFFFFFFFF, np.uint32)
    if blocks:
        ssm[:] = (np.arange(ssm.size).reshape(ssm.shape) + (1 << 31)).astype(np.uint32)
    t["req_ssm"] = ssm.reshape(-1)
    ctx.import_tables(t, {"cap_kv": a.n_kv, "cap_ssm": a.n_ssm, "gap_bytes": a.pool - a.n_kv * a.u_kv - a.n_ssm * a.u_ssm,
                          "last_rebalance_op": 0xFFFFFFFFFFFFFFFF})
    return ctx


def _classes(lengths):
    """Requests of like length together: index lists, so that padding at most doubles the plain form's work."""
    by = {}
    for i, v in enumerate(lengths):
        by.setdefault(max(0, v - 1).bit_length(), []).append(i)
    return [by[k] for k in sorted(by)]


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    perm = random.Random(seed)
    new, held = _plan(case)
    cu = torch.tensor([0] + new).cumsum(0).to(torch.int32)
    s = SimpleNamespace(case=case, new=new, held=held, dt=DT[case["dtype"]], n=case["n"], cu=cu.cuda(), total=int(cu[-1]),
                        starts=cu[:-1].long().cuda(), new_t=torch.tensor(new, device="cuda"))
    s.owner = torch.repeat_interleave(torch.arange(s.n, device="cuda"), s.new_t)         # list entry of each row
    s.reqs = torch.arange(s.n, dtype=torch.int32, device="cuda")
    return (_prepare_state if held is None else _prepare_attn)(s, case, gen, perm)


def _prepare_state(s, case, gen, perm):
    d, ns, w, g, nl = case["channels"], case["states"], case["width"], case["groups"], case["layers"]
    a = _arena(case, s.n + 1, s.n * nl + 2)
    s.arena = a
    # the blocks of the layer under test fill slots 1 .. n in some order; the other layers' lie around them
    mine = list(range(1, 1 + s.n))
    perm.shuffle(mine)
    it = iter([x for x in range(a.n_ssm) if not 1 <= x < 1 + s.n])
    blocks = [[mine[i] if l == case["layer"] else next(it) for l in range(nl)] for i in range(s.n)]
    end, u = a.pool // 4, a.u_ssm // 4
    # slot j lies at the end of the arena, j + 1 units back: row r of this view is slot n - r
    region = a.arena.view(torch.float32)[end - (1 + s.n) * u: end - u].view(s.n, u)
    region.normal_(generator=gen)
    s.state = region[:, : d * ns].unflatten(1, (d, ns))
    s.window = region[:, d * ns: d * (ns + w - 1)].unflatten(1, (w - 1, d))
    s.window.copy_(s.window.to(s.dt))                           # rows that came in earlier
    s.row = torch.tensor([s.n - m for m in mine], device="cuda")
    normal = lambda *shape, scale=1.0: torch.randn(*shape, device="cuda", generator=gen).mul_(scale)
    s.resume = None
    if case["op"].endswith("prompt"):
        s.resume = torch.tensor([case["resume"] * (i % 2) for i in range(s.n)], dtype=torch.int32, device="cuda")
    # the two halves of one projection: what goes in, and the gate
    both = torch.empty(s.total, 2 * d, dtype=s.dt, device="cuda").normal_(generator=gen)
    s.x, s.z = both[:, :d], both[:, d:]
    s.bias = normal(d, scale=0.3) if case["bias"] else None
    if case["op"].startswith("conv"):
        s.weight = normal(d, w, scale=w ** -0.5)
    else:
        s.u = torch.empty(s.total, d, dtype=s.dt, device="cuda").normal_(generator=gen).mul_(0.5)
        s.delta = torch.empty(s.total, d, dtype=s.dt, device="cuda").normal_(generator=gen).mul_(0.5)
        # B and C lie behind the low-rank steps in the rows of another projection
        rank = 8 * (-(-d // 128))
        bc = torch.empty(s.total, rank + 2 * g * ns, dtype=s.dt, device="cuda").normal_(generator=gen)
        s.b, s.c = (bc[:, rank + i * g * ns: rank + (i + 1) * g * ns] for i in (0, 1))
        # decays as such layers are made: rates 1 .. states, steps of 0.001 to 0.1 (the inverse of softplus as their bias)
        s.a = -torch.arange(1, ns + 1, device="cuda") * torch.exp(normal(d, ns, scale=0.2))
        step = torch.exp(torch.rand(d, device="cuda", generator=gen) * 4.6 - 6.9)
        s.bias = step + torch.log(-torch.expm1(-step)) if case["bias"] else None
        if s.bias is None:
            s.delta.add_(-4.0)
        s.skip = normal(d) if case["bias"] else None
    if s.resume is not None:
        s.classes = [(torch.tensor(idx, device="cuda"), max(s.new[i] for i in idx)) for idx in _classes(s.new)]
    if own:
        from paper_2605_22416_b200 import binding as B
        s.ctx = _handle(a, [1] * s.n, [[i] for i in range(s.n)], blocks)
        if case["op"].startswith("conv"):
            s.desc = B.conv_desc(channels=d, width=w, silu=True, dtype=s.dt, x_stride_bytes=4 * d)
        else:
            s.desc = B.scan_desc(channels=d, groups=g, states=ns, softplus=True, dtype=s.dt, z_stride_bytes=4 * d,
                                 b_stride_bytes=s.b.stride(0) * 2, c_stride_bytes=s.c.stride(0) * 2)
        if case["op"] == "scan_prompt":
            s.ws = torch.empty(max(16, s.ctx.scan_workspace_bytes(s.desc, s.n, s.total)), dtype=torch.uint8, device="cuda")
    return s


def _prepare_attn(s, case, gen, perm):
    T, hk, hq, d = case["page_tokens"], case["kv_heads"], case["q_heads"], case["head_dim"]
    pages = [-(-v // T) for v in s.held]
    n_kv = sum(pages) + 3
    slots = list(range(n_kv))
    perm.shuffle(slots)
    it = iter(slots)
    chains = [[next(it) for _ in range(p)] for p in pages]
    a = _arena(case, n_kv, 1)
    s.arena = a
    # all pages of the layer under test hold numbers; what lies behind the last token of a chain is left over from others
    s.kv = a.arena[: n_kv * a.u_kv].view(s.dt).view(n_kv, case["layers"], 2, T, hk, d)
    s.kv[:, case["layer"]].normal_(generator=gen)
    s.chain_t = [torch.tensor(c, device="cuda") for c in chains]
    s.held_t = torch.tensor(s.held, device="cuda")
    # place of each row in its chain
    s.at = torch.arange(s.total, device="cuda") + torch.repeat_interleave(s.held_t - s.new_t - s.starts, s.new_t)
    normal = lambda *shape, scale=1.0: torch.empty(*shape, dtype=s.dt, device="cuda").normal_(generator=gen).mul_(scale)
    if case["op"].startswith("rows"):
        qkv = normal(s.total, (hq + 2 * hk) * d, scale=1.5)               # rows of one projection
        s.q, s.k, s.v = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hk * d, hk * d], 1))
        s.wq, s.wk = ((1 + 0.2 * torch.randn(d, device="cuda", generator=gen)) if case["norm"] else None for _ in range(2))
        half = case["rotary"] // 2
        s.freq = (10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / max(1, half))).float() if half else None
        table = torch.zeros(s.n, max(pages), dtype=torch.long, device="cuda")
        for i, c in enumerate(s.chain_t):
            table[i, : len(c)] = c
        s.table = table
    else:
        s.q = normal(s.total, hq, d, scale=1.5)
        s.scale = 1.0 / math.sqrt(d)
        s.groups = []
        for idx in _classes(s.held):
            most = max(pages[i] for i in idx)
            t = torch.tensor([chains[i] + [0] * (most - pages[i]) for i in idx], device="cuda")
            s.groups.append((torch.tensor(idx, device="cuda"), t, max(s.held[i] for i in idx)))
    if own:
        from paper_2605_22416_b200 import binding as B
        s.ctx = _handle(a, s.held, chains, [])
        if case["op"].startswith("rows"):
            stride = s.q.stride(0) * 2
            s.desc = B.rows_desc(q_heads=hq, rotary_dim=case["rotary"], neighbours=case["neighbours"], eps=1e-6, dtype=s.dt,
                                 q_stride_bytes=stride, k_stride_bytes=stride, v_stride_bytes=stride)
        else:
            s.desc = B.attn_desc(q_heads=hq, dtype=s.dt, scale=s.scale)
            s.ws = torch.empty(max(16, s.ctx.attn_workspace_bytes(s.desc, s.n)), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------- the calls
def run(s):
    if own:
        return _run_own(s)
    return {"conv_prompt": _plain_conv, "conv_step": _plain_conv, "scan_prompt": _plain_scan_prompt, "scan_step": _plain_scan_step,
            "rows_prompt": _plain_rows, "rows_step": _plain_rows, "prompt": _plain_prompt, "decode": _plain_decode}[s.case["op"]](s)


def _run_own(s):
    c, op = s.case, s.case["op"]
    if op.startswith("conv"):
        out = torch.empty(s.total, c["channels"], dtype=s.dt, device="cuda")
        if op == "conv_prompt":
            s.ctx.conv_prompt(c["layer"], s.desc, s.reqs, s.n, s.cu, s.total, s.resume, s.x, s.weight, s.bias, out)
        else:
            s.ctx.conv_step(c["layer"], s.desc, s.reqs, s.n, s.x, s.weight, s.bias, out)
        return {"out": out, "window": s.window}
    if op.startswith("scan"):
        out = torch.empty_like(s.u)
        if op == "scan_prompt":
            s.ctx.scan_prompt(c["layer"], s.desc, s.reqs, s.n, s.cu, s.total, s.resume, s.u, s.delta, s.b, s.c, s.z, s.a, s.skip, s.bias, out,
                              s.ws, s.ws.numel())
        else:
            s.ctx.scan_step(c["layer"], s.desc, s.reqs, s.n, s.u, s.delta, s.b, s.c, s.z, s.a, s.skip, s.bias, out)
        return {"out": out, "state": s.state}
    out = torch.empty(s.total, c["q_heads"], c["head_dim"], dtype=s.dt, device="cuda")
    if op.startswith("rows"):
        if op == "rows_prompt":
            s.ctx.attn_rows_prompt(c["layer"], s.desc, s.reqs, s.n, s.cu, s.total, None, s.q, s.k, s.v, s.wq, s.wk, s.freq, out)
        else:
            s.ctx.attn_rows_step(c["layer"], s.desc, s.reqs, s.n, None, s.q, s.k, s.v, s.wq, s.wk, s.freq, out)
        return {"q": out, "kv": s.kv[:, c["layer"]]}
    lse = torch.empty(s.total, c["q_heads"], dtype=torch.float32, device="cuda")
    if op == "prompt":
        s.ctx.attn_window_prompt(c["layer"], s.desc, c["window"], c["sinks"], s.reqs, s.n, s.cu, s.total, s.q, out, lse, s.ws, s.ws.numel())
    else:
        s.ctx.attn_window_decode(c["layer"], s.desc, c["window"], c["sinks"], s.reqs, s.n, s.q, out, lse, s.ws, s.ws.numel())
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------- plain forms (32 bits)
def _fresh(s, first):
    """What the requests start from: zeros where nothing is continued."""
    if s.resume is None:
        return first
    keep = (s.resume != 0).view(-1, *[1] * (first.dim() - 1))
    return torch.where(keep, first, torch.zeros_like(first))


def _plain_conv(s):
    c = s.case
    d, w = c["channels"], c["width"]
    before = _fresh(s, s.window[s.row])                                      # [n, w - 1, d]
    x = s.x.float()
    place = torch.arange(s.total, device="cuda") - s.starts[s.owner]         # of a row in its request
    y = x * s.weight[:, w - 1]
    for back in range(1, w):
        old = torch.zeros_like(x)
        old[back:] = x[: s.total - back]
        edge = (place < back).nonzero().squeeze(1)
        old[edge] = before[s.owner[edge], w - 1 - back + place[edge]]
        y.addcmul_(old, s.weight[:, w - 1 - back])
        del old
    if s.bias is not None:
        y += s.bias
    y = y / (1 + (-y).exp())
    for j in range(w - 1):                                                   # the last w - 1 rows of each request
        p = s.new_t - (w - 1) + j
        there = (p >= 0)[:, None]
        s.window[s.row, j] = torch.where(there, x[(s.starts + p).clamp(0, s.total - 1)], before.gather(1, (p + w - 1).clamp(0, w - 2)[:, None, None].expand(-1, 1, d)).squeeze(1))
    return {"out": y.to(s.dt), "window": s.window}


def _softplus(x):
    return torch.where(x > 20, x, torch.log1p(x.clamp(max=20).exp()))


def _steps(s, rows=None):
    """Step sizes, inputs, gates of some rows, B and C by group: 32 bits."""
    c = s.case
    pick = (lambda t: t) if rows is None else (lambda t: t[rows])
    dl = pick(s.delta).float()
    if s.bias is not None:
        dl = dl + s.bias
    gr = (c["groups"], c["states"])
    return _softplus(dl), pick(s.u).float(), pick(s.b).float().unflatten(-1, gr), pick(s.c).float().unflatten(-1, gr)


def _finish(s, y, u, z):
    if s.skip is not None:
        y = y + s.skip * u
    z = z.float()
    return (y * (z / (1 + (-z).exp()))).to(s.dt)


def _plain_scan_step(s):
    c = s.case
    g, d, ns = c["groups"], c["channels"], c["states"]
    dl, u, b, cc = _steps(s)
    h = s.state[s.row]
    h *= (dl[..., None] * s.a).exp_()
    h.view(s.n, g, d // g, ns).add_((dl * u).view(s.n, g, d // g, 1) * b[:, :, None])
    s.state[s.row] = h
    y = (h.view(s.n, g, d // g, ns) * cc[:, :, None]).sum(-1).view(s.n, d)
    return {"out": _finish(s, y, u, s.z), "state": s.state}


def _plain_scan_prompt(s, piece=128):
    """Pieces of 128 tokens side by side, token by token: once from zero for the state that each leaves, then, with the states
    handed from piece to piece, for the outputs."""
    c = s.case
    g, d, ns = c["groups"], c["channels"], c["states"]
    out = torch.empty_like(s.u)
    before = _fresh(s, s.state[s.row])
    for idx, most in s.classes:
        p = min(piece, most)
        n, m = len(idx), -(-most // p)
        i = torch.arange(m * p, device="cuda")
        there = (i[None] < s.new_t[idx][:, None]).view(n, m, p)
        row = (s.starts[idx][:, None] + i[None]).clamp(max=s.total - 1).view(n, m, p)
        first = before[idx]

        def token(h, t, want):
            dl, u, b, cc = _steps(s, row[:, :, t])
            dl = dl * there[:, :, t, None]
            h *= (dl[..., None] * s.a).exp_()
            hg = h.view(n, m, g, d // g, ns)
            hg.addcmul_((dl * u).view(n, m, g, d // g, 1), b[:, :, :, None])
            if want:
                k = there[:, :, t]
                y = (hg * cc[:, :, :, None]).sum(-1).view(n, m, d)
                at = row[:, :, t][k]
                out[at] = _finish(s, y[k], u[k], s.z[at])
            return dl

        start = torch.zeros(n, m, d, ns, device="cuda")
        if m > 1:
            h = torch.zeros_like(start)
            sums = torch.zeros(n, m, d, device="cuda")
            for t in range(p):
                sums += token(h, t, False)
            cur = first
            for j in range(m):
                start[:, j] = cur
                cur = cur * (sums[:, j, :, None] * s.a).exp_() + h[:, j]
            del h
        else:
            start[:, 0] = first
        for t in range(p):
            token(start, t, True)
        s.state[s.row[idx]] = start[:, -1]           # rows behind a request's last change nothing
    return {"out": out, "state": s.state}


def _turn(x, cos, sin, neighbours):
    """Rotates the leading columns of x [rows, heads, dim] by pairs: (2i, 2i + 1), or (i, i + half)."""
    half = cos.shape[1]
    if half == 0:
        return x
    cos, sin = cos[:, None], sin[:, None]
    lead = x[..., : 2 * half]
    p, q = (lead[..., 0::2], lead[..., 1::2]) if neighbours else (lead[..., :half], lead[..., half:])
    a, b = p * cos - q * sin, q * cos + p * sin
    lead = torch.stack([a, b], -1).flatten(-2) if neighbours else torch.cat([a, b], -1)
    return torch.cat([lead, x[..., 2 * half:]], -1)


def _plain_rows(s):
    c = s.case
    if s.freq is None:
        cos = sin = torch.zeros(s.total, 0, device="cuda")
    else:
        angle = s.at.double()[:, None] * s.freq.double()          # far positions: angles in 64 bits
        cos, sin = angle.cos().float(), angle.sin().float()

    def one(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
        return _turn(x, cos, sin, c["neighbours"]).to(s.dt)

    slot, off = s.table[s.owner, s.at // c["page_tokens"]], s.at % c["page_tokens"]
    s.kv[slot, c["layer"], 0, off] = one(s.k, s.wk)
    s.kv[slot, c["layer"], 1, off] = s.v
    return {"q": one(s.q, s.wq), "kv": s.kv[:, c["layer"]]}


def _pages(s, table, part, valid):
    """K or V of the layer for a class of requests: [requests, heads, tokens, dim], zeros behind each length."""
    x = s.kv[table, s.case["layer"], part].flatten(1, 2)
    return torch.where(valid[:, :, None, None], x, x.new_zeros(())).permute(0, 2, 1, 3).float()


def _plain_decode(s):
    c = s.case
    hk, hq, d, w, sinks = c["kv_heads"], c["q_heads"], c["head_dim"], c["window"], c["sinks"]
    out = torch.empty_like(s.q)
    lse = torch.empty(s.n, hq, dtype=torch.float32, device="cuda")
    for idx, table, _ in s.groups:
        held = s.held_t[idx]
        pos = torch.arange(table.shape[1] * c["page_tokens"], device="cuda")
        valid = pos[None] < held[:, None]
        seen = valid & ((pos[None] >= held[:, None] - w) | (pos[None] < sinks))
        k, v = (_pages(s, table, part, valid) for part in (0, 1))
        p = (s.q[idx].float().view(len(idx), hk, hq // hk, d) @ k.transpose(2, 3)).mul_(s.scale).masked_fill_(~seen[:, None, None], -math.inf)
        top = p.amax(-1, keepdim=True)
        p = (p - top).exp()
        tot = p.sum(-1, keepdim=True)
        out[idx] = (p @ v / tot).reshape(len(idx), hq, d).to(s.dt)
        lse[idx] = (top + tot.log()).view(len(idx), hq)
    return {"out": out, "lse": lse}


def _plain_prompt(s):
    """Request by request, 512 rows at once over the keys that any of them sees."""
    c = s.case
    T, hk, hq, d, w, sinks = c["page_tokens"], c["kv_heads"], c["q_heads"], c["head_dim"], c["window"], c["sinks"]
    out = torch.empty_like(s.q)
    lse = torch.empty(s.total, hq, dtype=torch.float32, device="cuda")
    row = 0
    for r in range(s.n):
        past = s.held[r] - s.new[r]
        for a in range(0, s.new[r], 512):
            b = min(s.new[r], a + 512)
            low = max(0, past + a - w + 1)
            lead = min(low, sinks)
            j = torch.cat([torch.arange(lead, device="cuda"), torch.arange(low, past + b, device="cuda")])
            i = torch.arange(past + a, past + b, device="cuda")
            k, v = (s.kv[s.chain_t[r][j // T], c["layer"], part, j % T].float().transpose(0, 1) for part in (0, 1))      # [hk, keys, d]
            q = s.q[row + a: row + b].float().view(b - a, hk, hq // hk, d).permute(1, 2, 0, 3).reshape(hk, -1, d)
            p = (q @ k.transpose(1, 2)).mul_(s.scale).view(hk, hq // hk, b - a, len(j))
            p.masked_fill_((j > i[:, None]) | ((j <= i[:, None] - w) & (j >= sinks)), -math.inf)
            top = p.amax(-1, keepdim=True)
            p.sub_(top).exp_()
            tot = p.sum(-1, keepdim=True)
            o = (p.view(hk, -1, len(j)) @ v).view(hk, hq // hk, b - a, d) / tot
            out[row + a: row + b] = o.permute(2, 0, 1, 3).reshape(b - a, hq, d).to(s.dt)
            lse[row + a: row + b] = (top + tot.log()).squeeze(-1).permute(2, 0, 1).reshape(b - a, hq)
        row += s.new[r]
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------- 64 bits, from the definitions
def exact(case, seed):
    global own
    was, own = own, False           # the same inputs without the library's handle
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op.startswith("conv"):
        return _exact_conv(s)
    if op.startswith("scan"):
        return _exact_scan(s)
    return _exact_rows(s) if op.startswith("rows") else _exact_attn(s)


def _exact_conv(s):
    """Request by request: the row's last inputs one behind the other."""
    w = s.case["width"]
    out = torch.empty(s.total, s.case["channels"], dtype=torch.float64, device="cuda")
    window = s.window.double()
    at = 0
    for r in range(s.n):
        old = window[s.row[r]]
        if s.resume is not None and not int(s.resume[r]):
            old = torch.zeros_like(old)
        for a in range(0, s.new[r], 8192):          # the rows before it are the window of the next part
            b = min(s.new[r], a + 8192)
            line = torch.cat([old, s.x[at + a: at + b].double()])
            y = sum(line[j: j + b - a] * s.weight[:, j].double() for j in range(w))
            y = y if s.bias is None else y + s.bias.double()
            out[at + a: at + b] = y * torch.sigmoid(y)
            old = line[b - a:]
        window[s.row[r]] = old
        at += s.new[r]
    return {"out": out, "window": window}


def _exact_scan(s):
    """Token by token, all requests side by side; a request that has ended no longer changes."""
    c = s.case
    rep = c["channels"] // c["groups"]
    state = s.state.double()
    mine = state[s.row]
    if s.resume is not None:
        mine = mine * s.resume[:, None, None]
    out = torch.zeros(s.u.shape, dtype=torch.float64, device="cuda")
    order = sorted(range(s.n), key=lambda i: -s.new[i])
    o = torch.tensor(order, device="cuda")
    mine, starts, a = mine[o], s.starts[o], s.a.double()
    alive = s.n
    for t in range(s.new[order[0]]):
        while s.new[order[alive - 1]] <= t:
            alive -= 1
        at = starts[:alive] + t
        dl = s.delta[at].double()
        dl = torch.logaddexp(dl if s.bias is None else dl + s.bias, torch.zeros((), dtype=torch.float64, device="cuda"))
        b, cc = (x[at].double().unflatten(1, (c["groups"], c["states"])).repeat_interleave(rep, 1) for x in (s.b, s.c))
        u = s.u[at].double()
        cur = mine[:alive]
        cur *= torch.exp(dl[..., None] * a)
        cur += (dl * u)[..., None] * b
        out[at] = (cur * cc).sum(-1)
    for i in range(0, s.total, 8192):
        j = slice(i, i + 8192)
        z = s.z[j].double()
        y = out[j] if s.skip is None else out[j] + s.skip.double() * s.u[j].double()
        out[j] = y * z * torch.sigmoid(z)
    state[s.row[o]] = mine
    return {"out": out, "state": state}


def _exact_rows(s):
    """Pairs of columns as complex numbers, turned by position times frequency."""
    c = s.case
    kv = s.kv[:, c["layer"]].double()
    half = c["rotary"] // 2
    q_out = torch.empty(s.q.shape, dtype=torch.float64, device="cuda")

    def one(x, weight, place):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / c["head_dim"] + 1e-6) * weight.double()
        if half:
            i = torch.arange(half, device="cuda")
            re, im = (2 * i, 2 * i + 1) if c["neighbours"] else (i, i + half)
            turned = torch.complex(x[..., re], x[..., im]) * torch.polar(torch.ones_like(place)[:, None, None], (place[:, None] * s.freq.double())[:, None])
            x = x.clone()
            x[..., re], x[..., im] = turned.real, turned.imag
        return x

    at = 0
    for r in range(s.n):
        rows = slice(at, at + s.new[r])
        place = torch.arange(s.held[r] - s.new[r], s.held[r], device="cuda")
        q_out[rows] = one(s.q[rows], s.wq, place.double())
        page, off = s.chain_t[r][place // c["page_tokens"]], place % c["page_tokens"]
        kv[page, 0, off] = one(s.k[rows], s.wk, place.double())
        kv[page, 1, off] = s.v[rows].double()
        at += s.new[r]
    return {"q": q_out, "kv": kv}


def _exact_attn(s):
    c = s.case
    hk, hq, d, w, sinks = c["kv_heads"], c["q_heads"], c["head_dim"], c["window"], c["sinks"]
    rep = hq // hk
    out = torch.zeros(s.total, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s.total, hq, dtype=torch.float64, device="cuda")
    pages = s.kv[:, c["layer"]]
    row = 0
    for r in range(s.n):
        tokens = pages[s.chain_t[r]].transpose(1, 2).flatten(0, 1)[: s.held[r]]      # [held, 2, hk, d]
        past = s.held[r] - s.new[r]
        for a in range(0, s.new[r], 256):
            b = min(s.new[r], a + 256)
            i = torch.arange(past + a, past + b, device="cuda")[:, None]
            near = max(0, past + a + 1 - w)               # nothing between the sinks and here is seen by these rows
            keys = [x for x in range(min(sinks, near))] + list(range(near, past + b))
            j = torch.tensor(keys, device="cuda")
            hidden = ~((j <= i) & ((i - j < w) | (j < sinks)))
            kv = tokens[j].double()
            for h in range(hk):
                heads = slice(h * rep, h * rep + rep)
                z = torch.einsum("ihd,jd->ihj", s.q[row + a: row + b, heads].double(), kv[:, 0, h]) * s.scale
                z.masked_fill_(hidden[:, None], -math.inf)
                l = torch.logsumexp(z, -1)
                lse[row + a: row + b, heads] = l
                out[row + a: row + b, heads] = torch.einsum("ihj,jd->ihd", z.sub_(l[..., None]).exp_(), kv[:, 1, h])
        row += s.new[r]
    return {"out": out, "lse": lse}
