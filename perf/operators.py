"""Cases for the operators that compute on the two caches in place: attention over paged KV chains (whole prompts,
single tokens, single tokens behind a shared prefix) and the linear recurrence with a decay per head on the SSM state
blocks (whole prompts, single tokens).

`own` false: the plain form, elementary torch operations in 32 bits.  `own` true: the library's entry points.
Both work on the same arena: KV pages and state blocks lie at random physical slots and are reached through a table.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
NO_PREFIX = 0xFFFFFFFF


# ---------------------------------------------------------------- cases
def _attn(op, **kw):
    c = {"op": op, "dtype": "bf16", "page_tokens": 16, "kv_heads": 8, "q_heads": 32, "head_dim": 128, "layers": 4,
         "layer": 2, "len_seed": 1, "long_share": 0.0, "long_lo": 1, "long_hi": 1}
    c.update(kw)
    return c


def _ssm(op, **kw):
    c = {"op": op, "dtype": "bf16", "heads": 32, "groups": 1, "dk": 16, "dv": 64, "conv": 2048 * 3, "layers": 2, "layer": 1,
         "len_seed": 1, "long_share": 0.0, "long_lo": 1, "long_hi": 1}
    c.update(kw)
    return c


def listed():
    return [
        # a step that admits a full `pr1` batch: 32 short prompts of very different lengths, nothing held before
        _attn("prompt", name="prompt_pr1", n=32, lo=32, hi=512, past_lo=0, past_hi=0),
        # sessions that come back: each appends a turn of 256 to 2048 tokens to a chain that was kept between turns
        _attn("prompt", name="prompt_sessions", n=12, lo=256, hi=2048, past_lo=1, past_hi=8192, q_heads=64, dtype="f16", len_seed=2),
        # one prompt of the `mixed_long` kind beside three ordinary ones, one of them a single token
        _attn("prompt", name="prompt_long", n=4, lo=1, hi=900, past_lo=0, past_hi=0, long_share=0.25, long_lo=32749, long_hi=32749, len_seed=3),
        # decode step of a full `pr1` batch: everything fits the L2 cache, latency counts
        _attn("decode", name="decode_pr1", n=32, lo=48, hi=640, prefix=0),
        # decode step of the `scale` workload: 1024 running requests of a chat-like length spread
        _attn("decode", name="decode_scale", n=1024, lo=40, hi=2400, prefix=0, layers=9, layer=4, len_seed=4),
        # decode step of `mixed_long`: a fifth of the batch holds 16 to 64 thousand tokens
        _attn("decode", name="decode_mixed_long", n=128, lo=100, hi=4000, prefix=0, long_share=0.2, long_lo=16384, long_hi=65536, len_seed=5),
        # a burst of agents behind one system prompt
        _attn("decode", name="prefix_agents", n=256, lo=16, hi=384, prefix=2048, len_seed=6),
        # many questions about one long document
        _attn("decode", name="prefix_document", n=61, lo=1, hi=2000, prefix=40009, dtype="f16", len_seed=7),
        # the SSM layers of the `pr1` admission step
        _ssm("ssm_prompt", name="ssm_prompt_pr1", n=32, lo=32, hi=512, resume=0),
        # a long document and short prompts, half of them continued from a kept state
        _ssm("ssm_prompt", name="ssm_prompt_long", n=5, lo=1, hi=2000, heads=128, groups=8, conv=8192 * 3, long_share=0.2,
             long_lo=65521, long_hi=65521, resume=1, len_seed=8),
        # decode step of `pr1`, and of `scale` (one megabyte of state for each request)
        _ssm("ssm_step", name="ssm_step_pr1", n=32),
        _ssm("ssm_step", name="ssm_step_scale", n=1023, heads=256, groups=8, conv=16384 * 3),
    ]


def _logu(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prompt", "decode", "prefix", "ssm_prompt", "ssm_step"])
    seed, dtype = rng.randrange(1 << 30), rng.choice(["bf16", "f16"])
    if op.startswith("ssm"):
        dk, dv = rng.choice([16, 32, 64, 128]), rng.choice([32, 64, 128])
        groups = rng.choice([1, 2, 4, 8])
        heads = groups * rng.choice([1, 2, 3, 4, 8])
        kw = dict(dk=dk, dv=dv, groups=groups, heads=heads, dtype=dtype, conv=4 * rng.randint(1, 500), len_seed=seed)
        if op == "ssm_step":
            most = max(1, min(1023, (1 << 27) // (heads * dk * dv)))
            return _ssm(op, n=_logu(rng, 1, most), **kw)
        n = _logu(rng, 1, 40)
        most = max(2, min(65536, 200_000_000 // (n * heads * max(dv, dk))))
        lo = _logu(rng, 1, most)
        return _ssm(op, n=n, lo=lo, hi=_logu(rng, lo, most), resume=rng.randint(0, 1), **kw)
    kv_heads, head_dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    kw = dict(kv_heads=kv_heads, q_heads=kv_heads * rng.choice([1, 2, 3, 4, 8, 16]), head_dim=head_dim, dtype=dtype,
              page_tokens=rng.choice([16, 32, 64]), layers=2, layer=rng.randint(0, 1), len_seed=seed)
    if op == "prompt":
        n = _logu(rng, 1, 64)
        # within the largest listed case's products: n * new * held * q_heads * head_dim
        most = int(math.sqrt(1.2e12 / (n * kw["q_heads"] * head_dim)))
        lo = _logu(rng, 1, min(most, 16384))
        hi = _logu(rng, lo, min(most, 16384))
        return _attn("prompt", n=n, lo=lo, hi=hi, past_lo=0, past_hi=rng.choice([0, 1]) * _logu(rng, 1, min(most, 16384)), **kw)
    n = _logu(rng, 1, 1024)
    most = max(16, min(65536, 800_000_000 // (n * kv_heads * head_dim)))
    lo = _logu(rng, 1, most)
    return _attn("decode", n=n, lo=lo, hi=_logu(rng, lo, most), prefix=_logu(rng, 16, 40000) if op == "prefix" else 0, **kw)


def _lengths(case, lo, hi, salt=0):
    """The case's own ragged lengths, spread over the logarithm; a share of them (at least one) from the long range."""
    r = random.Random(case["len_seed"] * 7919 + salt)
    v = [_logu(r, lo, hi) for _ in range(case["n"])]
    if case["long_share"] > 0:
        for i in r.sample(range(case["n"]), max(1, round(case["long_share"] * case["n"]))):
            v[i] = _logu(r, case["long_lo"], case["long_hi"])
    return v


def _plan(case):
    """(new tokens, tokens held) of each request."""
    if case["op"] == "prompt":
        new = _lengths(case, case["lo"], case["hi"])
        r = random.Random(case["len_seed"] + 17)
        return new, [a + r.randint(case["past_lo"], case["past_hi"]) for a in new]
    if case["op"] == "decode":
        return [1] * case["n"], _lengths(case, case["lo"], case["hi"])
    if case["op"] == "ssm_prompt":
        return _lengths(case, case["lo"], case["hi"]), None
    return [1] * case["n"], None


def work(case):
    new, held = _plan(case)
    if held is not None:
        hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
        pre = case.get("prefix", 0)
        pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(new, held)) + sum(new) * pre
        return {"bytes": 2 * 2 * hk * d * (sum(held) + pre) + 2 * 2 * sum(new) * hq * d + 4 * sum(new) * hq,
                "flops": 4 * hq * d * pairs}
    h, g, dk, dv = case["heads"], case["groups"], case["dk"], case["dv"]
    tokens, state = sum(new), case["n"] * h * dk * dv
    reads = state if case["op"] == "ssm_step" or case["resume"] else 0
    # the recurrence as written: decay and update (3 per state element), read-out (2)
    return {"bytes": tokens * (2 * (2 * h * dv + 2 * g * dk) + 4 * h) + 4 * (state + reads), "flops": 5 * tokens * h * dk * dv}


# ---------------------------------------------------------------- inputs
def _arena(case, gen, n_kv, n_ssm):
    """Arena of n_kv pages and n_ssm blocks: pages grow from its base, block j ends j units before its end."""
    m = SimpleNamespace(n_attn_layers=case.get("layers", 1), n_ssm_layers=1, page_tokens=case.get("page_tokens", 16),
                        kv_heads=case.get("kv_heads", 1), head_dim=case.get("head_dim", 64), kv_elem_bytes=2,
                        ssm_state_elems=8192 * 16, ssm_conv_elems=8192 * 3, ssm_elem_bytes=4)
    if "dk" in case:
        m.n_attn_layers, m.n_ssm_layers, m.kv_heads = 1, case["layers"], 8
        m.ssm_state_elems, m.ssm_conv_elems = case["heads"] * case["dk"] * case["dv"], case["conv"]
    u_kv = m.n_attn_layers * 2 * m.page_tokens * m.kv_heads * m.head_dim * 2
    u_ssm = -(-4 * (m.ssm_state_elems + m.ssm_conv_elems) // 16) * 16
    pool = -(-(n_kv * u_kv + n_ssm * u_ssm) // 128) * 128
    arena = torch.empty(pool, dtype=torch.uint8, device="cuda")
    return SimpleNamespace(model=m, u_kv=u_kv, u_ssm=u_ssm, pool=pool, arena=arena, n_kv=n_kv, n_ssm=n_ssm)


def _handle(a, held, chains, blocks):
    """What a user of the library keeps beside the arena: a context whose tables hold these chains and blocks."""
    import numpy as np
    from paper_2605_22416_b200 import binding as B
    n = len(held)
    max_pages = max(len(c) for c in chains)
    ctx = B.Context(a.model, a.pool, 0.5, 16, max_requests=n, max_pages=max_pages, arena=a.arena, migration_enabled=False)
    lay = ctx.layout
    t = {}
    for p, (nm, cap, used) in enumerate((("kv", a.n_kv, [s for c in chains for s in c]), ("ssm", a.n_ssm, [s for b in blocks for s in b]))):
        v, used = int(lay.vid_space[p]), np.asarray(used, np.int64)
        vt, ow = np.full(v, 0xFFFFFFFF, np.uint32), np.full(v, 0xFFFFFFFF, np.uint32)
        vt[: len(used)], ow[used] = used, np.arange(len(used))      # ids in order of use, slots anywhere
        free = np.setdiff1d(np.arange(cap), used)
        t[f"slot_stack_{nm}"], t[f"vid_stack_{nm}"] = free.astype(np.uint32), np.arange(len(used), v).astype(np.uint32)
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
    stats = {"cap_kv": a.n_kv, "cap_ssm": a.n_ssm, "gap_bytes": a.pool - a.n_kv * a.u_kv - a.n_ssm * a.u_ssm,
             "last_rebalance_op": 0xFFFFFFFFFFFFFFFF}
    ctx.import_tables(t, stats)
    return ctx


def _normal(gen, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, device="cuda", generator=gen) * scale).to(dtype)


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
    s = SimpleNamespace(case=case, new=new, dt=DT[case["dtype"]])
    cu = torch.tensor([0] + new).cumsum(0).to(torch.int32)
    s.cu, s.total, s.n = cu.cuda(), int(cu[-1]), case["n"]
    s.starts = cu[:-1].long().cuda()
    s.new_t = torch.tensor(new, device="cuda")
    if held is None:
        return _prepare_ssm(s, case, gen, perm)
    T, hk, hq, d = case["page_tokens"], case["kv_heads"], case["q_heads"], case["head_dim"]
    s.prefix = case.get("prefix", 0)
    s.held = held
    all_held = held + ([s.prefix] if s.prefix else [])      # the prefix is a request slot of its own
    pages = [-(-v // T) for v in all_held]
    n_kv = sum(pages) + 3
    slots = list(range(n_kv))
    perm.shuffle(slots)
    it = iter(slots)
    chains = [[next(it) for _ in range(p)] for p in pages]
    a = _arena(case, gen, n_kv, 1)
    s.arena = a
    # all pages of the layer under test hold numbers; what lies behind the last token of a chain is left over from others
    s.kv = a.arena[: n_kv * a.u_kv].view(s.dt).view(n_kv, case["layers"], 2, T, hk, d)
    s.kv[:, case["layer"]].normal_(generator=gen)
    s.q = _normal(gen, s.total, hq, d, dtype=s.dt, scale=1.5)
    s.scale = 1.0 / math.sqrt(d)
    s.held_t = torch.tensor(held, device="cuda")
    s.chain_t = [torch.tensor(c, device="cuda") for c in chains]
    s.groups = []
    for idx in _classes(held):
        most = max(pages[i] for i in idx)
        table = torch.tensor([chains[i] + [0] * (most - pages[i]) for i in idx], device="cuda")
        s.groups.append((torch.tensor(idx, device="cuda"), table, max(new[i] for i in idx)))
    s.reqs = torch.arange(s.n, dtype=torch.int32, device="cuda")
    if own:
        from paper_2605_22416_b200 import binding as B
        s.ctx = _handle(a, all_held, chains, [])
        s.desc = B.attn_desc(q_heads=hq, dtype=s.dt, scale=s.scale)
        s.ws = torch.empty(max(16, s.ctx.attn_workspace_bytes(s.desc, s.n)), dtype=torch.uint8, device="cuda")
    return s


def _prepare_ssm(s, case, gen, perm):
    h, g, dk, dv = case["heads"], case["groups"], case["dk"], case["dv"]
    nl = case["layers"]
    a = _arena(case, gen, s.n + 1, s.n * nl + 2)
    s.arena = a
    # the blocks of the layer under test fill slots [lo, lo + n) in some order; the other layers' lie around them
    lo = 1
    mine = list(range(lo, lo + s.n))
    perm.shuffle(mine)
    rest = [x for x in range(a.n_ssm) if not lo <= x < lo + s.n]
    it = iter(rest)
    blocks = [[mine[i] if l == case["layer"] else next(it) for l in range(nl)] for i in range(s.n)]
    end = a.pool // 4
    u = a.u_ssm // 4
    f = a.arena.view(torch.float32)
    # slot j lies at the end of the arena, j + 1 units back: row r of this view is slot lo + n - 1 - r
    region = f[end - (lo + s.n) * u: end - lo * u].view(s.n, u)[:, : h * dk * dv]
    region.normal_(generator=gen)
    s.state = region.view(s.n, h, dv, dk)
    s.row = torch.tensor([lo + s.n - 1 - m for m in mine], device="cuda")
    s.q = _normal(gen, s.total, g, dk, dtype=s.dt, scale=1 / math.sqrt(dk))
    s.k = _normal(gen, s.total, g, dk, dtype=s.dt)
    s.v = _normal(gen, s.total, h, dv, dtype=s.dt, scale=0.3)
    # decay of a head: a step size of the token times a rate of the head, as such layers make it
    rate = torch.exp(torch.rand(h, device="cuda", generator=gen) * 2.77)
    step = torch.exp(torch.rand(s.total, h, device="cuda", generator=gen) * 4.6 - 6.9)
    s.g = -(step * rate)
    s.resume = None
    if case["op"] == "ssm_prompt":
        s.resume = torch.tensor([case["resume"] * (i % 2) for i in range(s.n)], dtype=torch.int32, device="cuda")
        s.classes = [(torch.tensor(idx, device="cuda"), max(s.new[i] for i in idx)) for idx in _classes(s.new)]
    s.reqs = torch.arange(s.n, dtype=torch.int32, device="cuda")
    if own:
        from paper_2605_22416_b200 import binding as B
        s.ctx = _handle(a, [1] * s.n, [[i] for i in range(s.n)], blocks)
        s.desc = B.ssm_desc(heads=h, groups=g, dk=dk, dv=dv, dtype=s.dt)
        if case["op"] == "ssm_prompt":
            s.ws = torch.empty(max(16, s.ctx.ssm_workspace_bytes(s.desc, s.n, s.total)), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------- the calls
def run(s):
    if own:
        return _run_own(s)
    return {"prompt": _plain_prompt, "decode": _plain_decode, "ssm_prompt": _plain_ssm_prompt, "ssm_step": _plain_ssm_step}[s.case["op"]](s)


def _run_own(s):
    c = s.case
    if c["op"] in ("prompt", "decode"):
        out = torch.empty_like(s.q)
        lse = torch.empty(s.total, c["q_heads"], dtype=torch.float32, device="cuda")
        if c["op"] == "prompt":
            s.ctx.attn_prompt(c["layer"], s.desc, s.reqs, s.n, s.cu, s.total, s.q, out, lse, s.ws, s.ws.numel())
        else:
            s.ctx.attn_decode(c["layer"], s.desc, s.reqs, s.n, s.n if s.prefix else NO_PREFIX, s.q, out, lse, s.ws, s.ws.numel())
        return {"out": out, "lse": lse}
    out = torch.empty_like(s.v)
    if c["op"] == "ssm_prompt":
        s.ctx.ssm_prompt(c["layer"], s.desc, s.reqs, s.n, s.cu, s.total, s.resume, s.q, s.k, s.v, s.g, out, s.ws, s.ws.numel())
    else:
        s.ctx.ssm_step(c["layer"], s.desc, s.reqs, s.n, s.q, s.k, s.v, s.g, out)
    return {"out": out, "state": s.state}


# ---------------------------------------------------------------- plain forms (32 bits)
def _pages(s, table, part, valid):
    """K or V of the layer for a class of requests: [requests, heads, tokens, dim], zeros behind each length."""
    x = s.kv[table, s.case["layer"], part].flatten(1, 2)
    return torch.where(valid[:, :, None, None], x, x.new_zeros(())).permute(0, 2, 1, 3).float()


def _plain_prompt(s):
    c = s.case
    hk, hq, d = c["kv_heads"], c["q_heads"], c["head_dim"]
    g = hq // hk
    out = torch.empty_like(s.q)
    lse = torch.empty(s.total, hq, dtype=torch.float32, device="cuda")
    for idx, table, q_most in s.groups:
        held, new = s.held_t[idx], s.new_t[idx]
        L = table.shape[1] * c["page_tokens"]
        pos = torch.arange(L, device="cuda")
        k, v = (_pages(s, table, part, pos[None] < held[:, None]) for part in (0, 1))
        part_len = max(1, min(q_most, (1 << 30) // (len(idx) * hq * L)))
        for q0 in range(0, q_most, part_len):      # as many queries at once as the scores have room for
            i = torch.arange(q0, min(q_most, q0 + part_len), device="cuda")
            there = i[None] < new[:, None]
            row = (s.starts[idx][:, None] + i[None]).clamp(max=s.total - 1)
            q = s.q[row].float().view(len(idx), len(i), hk, g, d).permute(0, 2, 3, 1, 4).reshape(len(idx), hk, g * len(i), d)
            p = (q @ k.transpose(2, 3)).view(len(idx), hk, g, len(i), L).mul_(s.scale)
            seen = pos[None, None] <= ((held - new)[:, None] + i[None])[:, :, None]
            p.masked_fill_(~seen[:, None, None], -math.inf)
            top = p.amax(-1, keepdim=True)
            p.sub_(top).exp_()
            tot = p.sum(-1, keepdim=True)
            o = (p.view(len(idx), hk, g * len(i), L) @ v).view(len(idx), hk, g, len(i), d) / tot
            out[row[there]] = o.permute(0, 3, 1, 2, 4).reshape(len(idx), len(i), hq, d)[there].to(s.dt)
            lse[row[there]] = (top + tot.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(len(idx), len(i), hq)[there]
    return {"out": out, "lse": lse}


def _plain_decode(s):
    c = s.case
    hk, hq, d = c["kv_heads"], c["q_heads"], c["head_dim"]
    g = hq // hk
    out = torch.empty_like(s.q)
    lse = torch.empty(s.n, hq, dtype=torch.float32, device="cuda")
    if s.prefix:
        kp, vp = (s.kv[s.chain_t[-1], c["layer"], part].flatten(0, 1)[: s.prefix].permute(1, 0, 2).float() for part in (0, 1))
    for idx, table, _ in s.groups:
        held = s.held_t[idx]
        pos = torch.arange(table.shape[1] * c["page_tokens"], device="cuda")
        valid = pos[None] < held[:, None]
        k, v = (_pages(s, table, part, valid) for part in (0, 1))
        q = s.q[idx].float().view(len(idx), hk, g, d)
        p = (q @ k.transpose(2, 3)).mul_(s.scale).masked_fill_(~valid[:, None, None], -math.inf)
        top = p.amax(-1, keepdim=True)
        if s.prefix:
            pp = (q.transpose(0, 1).reshape(hk, len(idx) * g, d) @ kp.transpose(1, 2)).view(hk, len(idx), g, s.prefix).transpose(0, 1) * s.scale
            top = torch.maximum(top, pp.amax(-1, keepdim=True))
            pp = (pp - top).exp()
        p = (p - top).exp()
        tot = p.sum(-1, keepdim=True)
        o = p @ v
        if s.prefix:
            tot = tot + pp.sum(-1, keepdim=True)
            o = o + (pp.transpose(0, 1).reshape(hk, len(idx) * g, s.prefix) @ vp).view(hk, len(idx), g, d).transpose(0, 1)
        out[idx] = (o / tot).reshape(len(idx), hq, d).to(s.dt)
        lse[idx] = (top + tot.log()).view(len(idx), hq)
    return {"out": out, "lse": lse}


def _plain_ssm_step(s):
    c = s.case
    rep = c["heads"] // c["groups"]
    q, k = (x.float().repeat_interleave(rep, 1) for x in (s.q, s.k))
    st = s.state[s.row] * s.g.exp()[:, :, None, None]
    st += s.v.float()[:, :, :, None] * k[:, :, None, :]
    s.state[s.row] = st
    return {"out": (st @ q[:, :, :, None]).squeeze(-1).to(s.dt), "state": s.state}


def _plain_ssm_prompt(s, piece=128):
    """The recurrence by pieces of 128 tokens: products inside a piece, states between pieces by a triangle of decays."""
    c = s.case
    h, g, dk, dv = c["heads"], c["groups"], c["dk"], c["dv"]
    rep = h // g
    out = torch.empty_like(s.v)
    for idx, most in s.classes:
        n, m = len(idx), -(-most // piece)
        i = torch.arange(m * piece, device="cuda")
        there = i[None] < s.new_t[idx][:, None]
        row = (s.starts[idx][:, None] + i[None]).clamp(max=s.total - 1)
        keep = there[:, :, None]
        q, k = ((x[row].float() * keep[..., None]).view(n, m, piece, g, dk).permute(0, 3, 1, 2, 4) for x in (s.q, s.k))
        v = (s.v[row].float() * keep[..., None]).view(n, m, piece, h, dv).permute(0, 3, 1, 2, 4)
        # angles of far tokens: decays are summed in 64 bits, their differences are short again
        run = (s.g[row].double() * keep).view(n, m, piece, h).permute(0, 3, 1, 2).cumsum(-1)
        low = torch.ones(piece, piece, dtype=torch.bool, device="cuda").tril()
        decay = (run[..., :, None] - run[..., None, :]).float().masked_fill_(~low, -math.inf).exp_()
        sc = (q @ k.transpose(-1, -2)).repeat_interleave(rep, 1) * decay
        del decay
        y = sc @ v
        del sc
        tail = (run[..., -1:] - run).float().exp()
        k, q = k.repeat_interleave(rep, 1), q.repeat_interleave(rep, 1)
        local = (v * tail[..., None]).transpose(-1, -2) @ k                      # [n, h, m, dv, dk]
        first = s.state[s.row[idx]] * s.resume[idx][:, None, None, None]
        whole = torch.cat([torch.zeros_like(run[:, :, :1, 0]), run[..., -1]], -1).cumsum(-1)
        tri = torch.ones(m + 1, m + 1, dtype=torch.bool, device="cuda").tril()
        w = (whole[..., :, None] - whole[..., None, :]).float().masked_fill_(~tri, -math.inf).exp_()
        states = (w @ torch.cat([first[:, :, None], local], 2).flatten(3)).view(n, h, m + 1, dv, dk)
        y += (q * run.float().exp()[..., None]) @ states[:, :, :-1].transpose(-1, -2)
        out[row[there]] = y.permute(0, 2, 3, 1, 4).reshape(n, m * piece, h, dv)[there].to(s.dt)
        s.state[s.row[idx]] = states[:, :, -1]
    return {"out": out, "state": s.state}


# ---------------------------------------------------------------- 64 bits, from the definitions
def exact(case, seed):
    s = prepare_plain(case, seed)
    return (_exact_attn if "q_heads" in case else _exact_ssm)(s)


def prepare_plain(case, seed):
    """The same inputs without the library's handle."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _exact_attn(s):
    c = s.case
    hk, hq, d = c["kv_heads"], c["q_heads"], c["head_dim"]
    rep = hq // hk
    out = torch.zeros(s.total, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s.total, hq, dtype=torch.float64, device="cuda")
    pages = s.kv[:, c["layer"]]
    lead = pages[s.chain_t[-1]].transpose(1, 2).flatten(0, 1)[: s.prefix] if s.prefix else None
    row = 0
    for r in range(s.n):
        tokens = pages[s.chain_t[r]].transpose(1, 2).flatten(0, 1)[: s.held[r]]      # [held, 2, hk, d]
        if lead is not None:
            tokens = torch.cat([lead, tokens])
        past = len(tokens) - s.new[r]
        for kvh in range(hk):
            K, V = tokens[:, 0, kvh].double(), tokens[:, 1, kvh].double()
            heads = slice(kvh * rep, kvh * rep + rep)
            block = max(1, (1 << 27) // (rep * len(tokens)))
            for a in range(0, s.new[r], block):
                b = min(s.new[r], a + block)
                Q = s.q[row + a: row + b, heads].double()
                end = past + b
                z = torch.einsum("ihd,jd->ihj", Q, K[:end]) * s.scale
                if b - a > 1:
                    j, i = torch.arange(end, device="cuda"), torch.arange(past + a, end, device="cuda")
                    z.masked_fill_((j[None] > i[:, None])[:, None], -math.inf)
                l = torch.logsumexp(z, -1)
                lse[row + a: row + b, heads] = l
                out[row + a: row + b, heads] = torch.einsum("ihj,jd->ihd", z.sub_(l[..., None]).exp_(), V[:end])
        row += s.new[r]
    return {"out": out, "lse": lse}


def _exact_ssm(s):
    """Token by token, all requests side by side; a request that has ended no longer changes."""
    c = s.case
    rep = c["heads"] // c["groups"]
    if max(s.new) > 70_000:
        return None
    state = s.state.double()
    mine = state[s.row]
    if s.resume is not None:
        mine = mine * s.resume[:, None, None, None]
    out = torch.zeros(s.v.shape, dtype=torch.float64, device="cuda")
    order = sorted(range(s.n), key=lambda i: -s.new[i])
    o = torch.tensor(order, device="cuda")
    mine, starts = mine[o], s.starts[o]
    lengths = [s.new[i] for i in order]
    alive = s.n
    for t in range(lengths[0]):
        while lengths[alive - 1] <= t:
            alive -= 1
        at = starts[:alive] + t
        cur = mine[:alive]
        cur *= s.g[at].double().exp()[:, :, None, None]
        cur += s.v[at].double()[..., None] * s.k[at].double().repeat_interleave(rep, 1)[:, :, None]
        out[at] = torch.einsum("nhvk,nhk->nhv", cur, s.q[at].double().repeat_interleave(rep, 1))
    state[s.row[o]] = mine
    return {"out": out, "state": state}
