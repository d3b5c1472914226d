"""Performance cases of the operators around the quantized linears of a decoder layer: rotary positions, the paged
key / value cache with its block tables and slot maps, and the attention of new tokens over that cache.

``listed()`` and ``draw(rng)`` give cases, ``prepare(case, seed)`` the tensors a caller holds before a call,
``run(state)`` one call: with ``own`` set through the library's entry points, otherwise in elementary torch operations
in 32 bits, rounded once at the end.  ``exact(case, seed)`` computes the same outputs from the definitions in 64 bits.

Notation: B requests; request b has ctx[b] tokens in the cache and adds new[b]; T = sum of new; a page holds
`page` tokens; H query heads share Hkv key / value heads (head h reads key head h // (H / Hkv)); D = head size.
"""
import math
import random

import torch

own = False
DEV = "cuda"
_TWO64 = 1 << 64


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    heads = dict(heads=32, kv_heads=32, dim=128)         # the 7B-shaped layers (4096 = 32 x 128)
    heads13 = dict(heads=40, kv_heads=40, dim=128)       # the 13B-shaped layers (5120 = 40 x 128)
    heads33 = dict(heads=52, kv_heads=52, dim=128)       # the 33B-shaped layers (6656 = 52 x 128)
    shared = dict(heads=32, kv_heads=8, dim=128)         # four query heads to a key head
    return [
        # one decode step of a small server: eight requests, one token each; latency is all that counts
        dict(name="plan decode 8", op="plan", reqs=8, ctx_lo=40, ctx_hi=4000, new_lo=1, new_hi=1, chunks=0, chunk=0,
             page=16, release=0, slack=0, lens=1),
        # one step of a large server: 512 requests decode, some start with a long prompt, some end and give pages back,
        # the token buffer has unused rows
        dict(name="plan mixed 512", op="plan", reqs=512, ctx_lo=0, ctx_hi=8000, new_lo=1, new_hi=1, chunks=9, chunk=1777,
             page=16, release=31, slack=77, lens=2),
        # fine-tuning step, 2048 tokens = 4 x 512, forward
        dict(name="rope train fwd 2048", op="rope", tokens=2048, seq=512, start=0, rotary=128, layout="half", inverse=False,
             dtype="bf16", fused=False, scale="none", **heads),
        # its backward on fp32 gradients, 8 sequences of uneven total length, pairs side by side, part of the head
        dict(name="rope train bwd 8191", op="rope", tokens=8191, seq=1024, start=0, rotary=64, layout="pairs", inverse=True,
             dtype="f32", fused=False, scale="none", **heads13),
        # one token of one request, far into a context stretched to eight times its trained length
        dict(name="append 1 token", op="append", tokens=1, seq=1, start=30001, rotary=128, layout="half", dtype="bf16",
             fused=True, scale="banded", page=16, **shared),
        # a prompt chunk written into the cache
        dict(name="append chunk 4095", op="append", tokens=4095, seq=4095, start=1, rotary=128, layout="half", dtype="bf16",
             fused=False, scale="linear", page=64, **heads33),
        # a lone user decoding: the latency case
        dict(name="attend 1 x 513", op="attend", reqs=1, ctx_lo=512, ctx_hi=512, new_lo=1, new_hi=1, chunks=0, chunk=0,
             page=16, window=0, lens=1, **shared),
        # a busy server: 64 requests of very uneven length decode, shared key heads
        dict(name="attend decode 64 shared", op="attend", reqs=64, ctx_lo=30, ctx_hi=8100, new_lo=1, new_hi=1, chunks=0,
             chunk=0, page=16, window=0, lens=2, **shared),
        # long contexts, every query head its own keys: pure cache bandwidth
        dict(name="attend decode 6 x 16k", op="attend", reqs=6, ctx_lo=14000, ctx_hi=16300, new_lo=1, new_hi=1, chunks=0,
             chunk=0, page=64, window=0, lens=3, **heads13),
        # a few drafted tokens per request are checked at once
        dict(name="attend verify 16 x 5", op="attend", reqs=16, ctx_lo=700, ctx_hi=4000, new_lo=3, new_hi=7, chunks=0,
             chunk=0, page=32, window=0, lens=4, **shared),
        # one step that mixes decoding requests with two prompt chunks, one of them a fresh prompt
        dict(name="attend mixed 16", op="attend", reqs=16, ctx_lo=0, ctx_hi=3000, new_lo=1, new_hi=1, chunks=2, chunk=1021,
             page=16, window=0, lens=5, **heads),
        # a long document is read in chunks: 4096 new tokens behind 28k cached ones; tensor-core work
        dict(name="attend chunk 4096 at 28k", op="attend", reqs=1, ctx_lo=28000, ctx_hi=28000, new_lo=4096, new_hi=4096,
             chunks=0, chunk=0, page=64, window=0, lens=6, **heads13),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["plan", "rope", "append", "attend", "attend", "attend"])
    lens = rng.randrange(1 << 30)
    kv = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    heads = kv * rng.choice([g for g in (1, 1, 2, 3, 4, 5, 7, 8, 16) if g * kv <= 64])
    dim = rng.choice([64, 128, 128, 128])
    page = rng.choice([16, 16, 32, 64, 128])
    h = dict(heads=heads, kv_heads=kv, dim=dim)
    if op == "plan":
        reqs = _log_int(rng, 1, 512)
        return dict(op=op, reqs=reqs, ctx_lo=0, ctx_hi=_log_int(rng, 10, 8000), new_lo=1, new_hi=rng.choice([1, 1, 5]),
                    chunks=min(reqs, rng.randrange(9)), chunk=_log_int(rng, 20, 1700), page=page,
                    release=rng.randrange(1 + reqs // 16), slack=rng.randrange(64), lens=lens)
    if op in ("rope", "append"):
        tokens = _log_int(rng, 1, 4000)
        rotary = rng.choice([dim, dim, dim // 2])
        c = dict(op=op, tokens=tokens, seq=max(1, tokens // rng.choice([1, 2, 5])), start=_log_int(rng, 1, 100000) - 1,
                 rotary=rotary, layout=rng.choice(["half", "pairs"]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                 fused=rng.random() < 0.5, scale=rng.choice(["none", "linear", "banded"]), **h)
        return dict(c, page=page) if op == "append" else dict(c, inverse=rng.random() < 0.5)
    # kept below the largest listed case: at most 1e9 scores over the padded batch, at most 2 GB of keys and values
    kind = rng.choice(["decode", "decode", "verify", "chunk", "mixed"])
    hi = _log_int(rng, 20, 16000)
    reqs = {"decode": _log_int(rng, 1, 64), "verify": _log_int(rng, 1, 32), "chunk": rng.choice([1, 1, 2]),
            "mixed": _log_int(rng, 2, 16)}[kind]
    new_lo, new_hi = {"decode": (1, 1), "verify": (2, 9), "chunk": (0, 0), "mixed": (1, 1)}[kind]
    chunks = {"decode": 0, "verify": 0, "chunk": reqs, "mixed": 1}[kind]
    chunk = _log_int(rng, 20, 2500) if chunks else 0
    most = max(new_hi, chunk)
    hi = max(1, min(hi, int(1e9 / (reqs * most * heads)) - most, int(1e9 / (reqs * kv * dim * 2)) - most))
    return dict(op=op, reqs=reqs, ctx_lo=rng.choice([0, hi // 2, hi]), ctx_hi=hi, new_lo=new_lo, new_hi=new_hi,
                chunks=chunks, chunk=chunk, page=page, window=rng.choice([0, 0, 0, 1000]), lens=lens, **h)


# ------------------------------------------------------------------------------------------------------------ inputs
def _lengths(c):
    """(ctx, new) of each request: a property of the case, equal for all seeds.  The first `chunks` requests bring a chunk."""
    r = random.Random(c["lens"])
    ctx = [r.randint(c["ctx_lo"], c["ctx_hi"]) for _ in range(c["reqs"])]
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["reqs"])]
    for b in range(c["chunks"]):
        new[b] = c["chunk"]
        if b % 2 == 1:
            ctx[b] = 0                       # every second chunk is the start of a prompt
    order = list(range(c["reqs"]))
    r.shuffle(order)
    return [ctx[b] for b in order], [new[b] for b in order]


def _pages(tokens, page):
    return -(-tokens // page)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + 13)


def _randn(g, *shape, dtype=torch.bfloat16, gain=1.0):
    """Normal values of the given type, drawn in pieces so that no 32-bit copy of a large cache exists."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    for piece in out.view(-1).split(1 << 26):
        piece.copy_(torch.randn(piece.shape, generator=g, device=DEV) * gain)
    return out


def _turns(rotary, scale, base=10000.0):
    """Rotation per position of each pair, in turns, before any rounding to the table's type."""
    f = [base ** (-2.0 * j / rotary) / (2.0 * math.pi) for j in range(rotary // 2)]
    if scale == "linear":                    # positions squeezed by four
        f = [v / 4.0 for v in f]
    elif scale == "banded":                  # slow pairs squeezed by eight, fast ones kept, a ramp between
        ramp = lambda v: min(1.0, max(0.0, (4096 * v - 1.0) / (32.0 - 1.0)))  # noqa: E731
        f = [v * ramp(v) + v / 8.0 * (1.0 - ramp(v)) for v in f]
    return f


def _table(rotary, scale):
    """The rotation table a caller keeps for a model: turns per position in units of 2^-64, as int64."""
    whole = [int(v * _TWO64) for v in _turns(rotary, scale)]
    return torch.tensor([w - _TWO64 if w >= _TWO64 // 2 else w for w in whole], dtype=torch.int64, device=DEV)


def _plan_inputs(c, seed):
    ctx, new = _lengths(c)
    reqs, page = c["reqs"], c["page"]
    g = _generator(seed)
    width = max(_pages(a + n, page) for a, n in zip(ctx, new)) + 3
    held = [_pages(a, page) for a in ctx]
    grow = sum(_pages(a + n, page) - h for a, n, h in zip(ctx, new, held))
    n_pages = sum(held) + grow + 40
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((reqs, width), -1, dtype=torch.int32, device=DEV)
    at = torch.cumsum(_i32(held), 0) - _i32(held)
    col = torch.arange(width, device=DEV)
    have = col[None] < _i32(held)[:, None]
    table[have] = perm[(at[:, None] + col[None])[have].long()]
    stack = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    n_free = n_pages - sum(held)
    stack[:n_free] = perm[sum(held):]
    release = torch.zeros(reqs, dtype=torch.int32, device=DEV)
    if c["release"]:
        release[torch.randperm(reqs, generator=g, device=DEV)[:c["release"]]] = 1
    return dict(ctx=_i32(ctx), new=_i32(new), release=release, table=table, stack=stack, count=_i32([n_free]),
                capacity=sum(new) + c["slack"], n_pages=n_pages)


def _rope_inputs(c, seed):
    g = _generator(seed)
    T, H, Hkv, D = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
    dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    if c["fused"]:                           # one tensor from one product, read through strides
        qkv = _randn(g, T, H + 2 * Hkv, D, dtype=dtype)
        q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    else:
        q, k, v = (_randn(g, T, n, D, dtype=dtype) for n in (H, Hkv, Hkv))
    at = torch.arange(T, device=DEV)
    return q, k, v, (c["start"] + at % c["seq"]).to(torch.int32), _table(c["rotary"], c["scale"])


def _cache_inputs(c, seed):
    """Cache, block tables and queries of an attention case."""
    ctx, new = _lengths(c)
    page, H, Hkv, D = c["page"], c["heads"], c["kv_heads"], c["dim"]
    g = _generator(seed)
    total = [a + n for a, n in zip(ctx, new)]
    need = [_pages(t, page) for t in total]
    n_pages = sum(need) + 7
    cache_k = _randn(g, n_pages, page, Hkv, D)
    cache_v = _randn(g, n_pages, page, Hkv, D)
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    width = max(need) + 1
    col = torch.arange(width, device=DEV)
    at = torch.cumsum(_i32(need), 0) - _i32(need)
    have = col[None] < _i32(need)[:, None]
    table = torch.zeros((c["reqs"], width), dtype=torch.int32, device=DEV)
    table[have] = perm[(at[:, None] + col[None])[have].long()]
    q = _randn(g, sum(new), H, D, gain=1.5)  # scores of standard deviation 1.5, as after a trained projection
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return dict(k=cache_k, v=cache_v, table=table, q=q, cu=_i32(cu), kv=_i32(total), new=new, total=total)


def prepare(c, seed):
    s = dict(case=c)
    if c["op"] == "plan":
        s.update(_plan_inputs(c, seed))
        T, B = s["capacity"], c["reqs"]
        new = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)  # noqa: E731
        s["outs"] = (new(B + 1), new(B), new(T), new(T), new(B), new(1))
    elif c["op"] in ("rope", "append"):
        s["q"], s["k"], s["v"], s["pos"], s["turns"] = _rope_inputs(c, seed)
        T, H, Hkv, D = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        if c["op"] == "append":
            n_pages = _pages(T, c["page"]) + 5
            g = _generator(seed + 1)
            s["slots"] = torch.randperm(n_pages, generator=g, device=DEV)[:_pages(T, c["page"])]
            at = torch.arange(T, device=DEV)
            s["slots"] = (s["slots"][at // c["page"]] * c["page"] + at % c["page"]).to(torch.int32)
            s["ck"], s["cv"] = (torch.zeros(n_pages, c["page"], Hkv, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
            s["oq"] = torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV)
        else:
            s["oq"], s["ok"] = (torch.empty(T, n, D, dtype=s["q"].dtype, device=DEV) for n in (H, Hkv))
    else:
        s.update(_cache_inputs(c, seed))
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
        s["scratch"] = {}                    # the workspace a caller keeps between its calls
    return s


# --------------------------------------------------------------------------------------------------------------- run
def run(s):
    return (_run_own if own else _run_plain)[s["case"]["op"]](s)


def _own_plan(s):
    from paper_2407_17029_b200 import binding as qb
    p = qb.kv_plan(s["ctx"], s["new"], s["table"], s["stack"], s["count"], s["case"]["page"], s["capacity"],
                   release=s["release"], outs=s["outs"])
    return dict(table=s["table"], stack=s["stack"], cu_new=p.cu_new, kv_len=p.kv_len, positions=p.positions, slots=p.slots,
                admitted=p.admitted, free_count=p.free_count)


def _own_cfg(s, qb):
    c = s["case"]
    return qb.Rope(c["dim"], c["rotary"], qb.ROPE_HALF if c["layout"] == "half" else qb.ROPE_PAIRS, s["turns"])


def _own_rope(s):
    from paper_2407_17029_b200 import binding as qb
    q, k = qb.rope(_own_cfg(s, qb), s["pos"], s["q"], s["k"], inverse=s["case"]["inverse"], out_q=s["oq"], out_k=s["ok"])
    return dict(q=q, k=k)


def _own_append(s):
    from paper_2407_17029_b200 import binding as qb
    q = qb.rope_append(_own_cfg(s, qb), s["pos"], s["slots"], s["q"], s["k"], s["v"], qb.KVCache(s["ck"], s["cv"]),
                       out_q=s["oq"])
    return dict(q=q, k=s["ck"], v=s["cv"])


def _own_attend(s):
    from paper_2407_17029_b200 import binding as qb
    cache = qb.KVCache(s["k"], s["v"])
    if "ws" not in s["scratch"]:
        s["scratch"]["ws"] = qb.alloc_attention_workspace(cache, s["q"])
    out, lse = qb.paged_attention(s["q"], cache, s["table"], s["cu"], s["kv"], window=s["case"]["window"], out=s["out"],
                                  lse=s["lse"], ws=s["scratch"]["ws"])
    return dict(out=out, lse=lse)


def _plain_plan(s):
    c = s["case"]
    page, T = c["page"], s["capacity"]
    B, width = s["table"].shape
    ctx, new, table, stack = s["ctx"].long(), s["new"].long(), s["table"], s["stack"]
    gone = s["release"] != 0
    held = (ctx + page - 1) // page
    back = torch.where(gone, held, torch.zeros_like(held))
    valid = ~gone & (ctx >= 0) & (new >= 0) & (ctx + new <= width * page)
    zero = torch.zeros_like(ctx)
    need = torch.where(valid, (ctx + new + page - 1) // page - held, zero)
    asked = torch.where(valid, new, zero)
    n_free = s["count"].long()
    pushed_end = torch.cumsum(back, 0)
    # pages given back go onto the stack in request order
    col = torch.arange(width, device=DEV)
    give = col[None] < back[:, None]
    place = torch.where(give, n_free + (pushed_end - back)[:, None] + col[None], torch.full_like(give, stack.numel(), dtype=torch.int64))
    wide = torch.cat([stack, stack.new_zeros(1)])
    wide.scatter_(0, place.reshape(-1), table.reshape(-1))
    stack.copy_(wide[:-1])
    avail = n_free + pushed_end[-1:]
    ok = valid & (torch.cumsum(need, 0) <= avail) & (torch.cumsum(asked, 0) <= T)
    need, asked = torch.where(ok, need, zero), torch.where(ok, asked, zero)
    end = torch.cumsum(need, 0)
    nth = (end - need)[:, None] + col[None] - held[:, None]
    fresh = (col[None] >= held[:, None]) & (col[None] < (held + need)[:, None])
    pick = torch.where(fresh, avail - 1 - nth, torch.zeros_like(nth))
    table.copy_(torch.where(fresh, stack[pick], table))
    cu = torch.cat([zero[:1], torch.cumsum(asked, 0)])
    t = torch.arange(T, device=DEV)
    real = t < cu[-1]
    b = torch.clamp(torch.searchsorted(cu[1:], t, right=True), max=B - 1)
    pos = torch.where(real, ctx[b] + t - cu[b], torch.zeros_like(t))
    slot = torch.where(real, table[b, torch.clamp(pos // page, max=width - 1)].long() * page + pos % page, torch.full_like(t, -1))
    kv = torch.where(gone, zero, ctx + asked)
    cast = lambda x: x.to(torch.int32)  # noqa: E731
    return dict(table=table, stack=stack, cu_new=cast(cu), kv_len=cast(kv), positions=cast(pos), slots=cast(slot),
                admitted=cast(ok), free_count=cast(avail - end[-1:]))


def _plain_rotate(x, pos, turns, rotary, layout, sign):
    """The rotation in 32 bits.  The phase is whole-number arithmetic: position x turns modulo one turn in 2^-64 units,
    of which the upper 32 bits become the angle."""
    phase = (pos.long()[:, None] * turns[None]) >> 32
    angle = phase.to(torch.float32) * (math.pi / 2.0 ** 31)
    co, si = torch.cos(angle)[:, None], torch.sin(angle)[:, None] * sign
    y = x.to(torch.float32)
    r = y[..., :rotary]
    if layout == "half":
        a, b = r[..., :rotary // 2], r[..., rotary // 2:]
        turned = torch.cat([a * co - b * si, b * co + a * si], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        turned = torch.stack([a * co - b * si, b * co + a * si], -1).flatten(-2)
    return torch.cat([turned, y[..., rotary:]], -1)


def _plain_rope(s):
    c = s["case"]
    sign = -1.0 if c["inverse"] else 1.0
    return dict(q=_plain_rotate(s["q"], s["pos"], s["turns"], c["rotary"], c["layout"], sign).to(s["q"].dtype),
                k=_plain_rotate(s["k"], s["pos"], s["turns"], c["rotary"], c["layout"], sign).to(s["k"].dtype))


def _plain_append(s):
    c = s["case"]
    q = _plain_rotate(s["q"], s["pos"], s["turns"], c["rotary"], c["layout"], 1.0).to(torch.bfloat16)
    k = _plain_rotate(s["k"], s["pos"], s["turns"], c["rotary"], c["layout"], 1.0).to(torch.bfloat16)
    at = s["slots"].long()
    s["ck"].view(-1, c["kv_heads"], c["dim"])[at] = k
    s["cv"].view(-1, c["kv_heads"], c["dim"])[at] = s["v"].to(torch.bfloat16)
    return dict(q=q, k=s["ck"], v=s["cv"])


def _plain_attend(s):
    c = s["case"]
    B, H, Hkv, D, page = c["reqs"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    G, N, L = H // Hkv, max(s["new"]), max(s["total"])
    cu, kv = s["cu"].long(), s["kv"].long()
    new = cu[1:] - cu[:-1]
    # queries padded to [B][Hkv][N * G][D], keys and values gathered to [B][Hkv][L][D]
    i = torch.arange(N, device=DEV)
    at = torch.clamp(cu[:-1, None] + i[None], max=s["q"].shape[0] - 1)
    q = s["q"][at].to(torch.float32).view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    slots = s["table"][:, :_pages(L, page)].long()
    keys = s["k"][slots].flatten(1, 2)[:, :L].permute(0, 2, 1, 3).to(torch.float32)
    score = (q @ keys.transpose(-1, -2)).mul_(1.0 / math.sqrt(D)).view(B, Hkv, N, G, L)
    del keys
    p = kv[:, None] - new[:, None] + i[None]                                   # position of each query
    j = torch.arange(L, device=DEV)
    seen = (j[None, None] <= p[..., None]) & (j[None, None] < kv[:, None, None])
    if c["window"]:
        seen &= j[None, None] > p[..., None] - c["window"]
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    w = score.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    vals = s["v"][slots].flatten(1, 2)[:, :L].permute(0, 2, 1, 3).to(torch.float32)
    o = (w.view(B, Hkv, N * G, L) @ vals).view(B, Hkv, N, G, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (torch.log(total) + top).squeeze(-1)
    real = (i[None] < new[:, None])
    back = lambda x: x.permute(0, 2, 1, 3, *range(4, x.dim())).flatten(2, 3)[real]  # noqa: E731
    return dict(out=back(o).to(torch.bfloat16), lse=back(lse))


_run_own = dict(plan=_own_plan, rope=_own_rope, append=_own_append, attend=_own_attend)
_run_plain = dict(plan=_plain_plan, rope=_plain_rope, append=_plain_append, attend=_plain_attend)


# -------------------------------------------------------------------------------------------------------------- work
def _visible(c):
    """(keys read by a request, query-key pairs) of each request."""
    ctx, new = _lengths(c)
    got = []
    for a, n in zip(ctx, new):
        w = c["window"] or (a + n + 1)
        pairs = sum(min(a + i + 1, w) for i in range(n))
        got.append((a + n - max(0, a + 1 - w) if n else 0, pairs))
    return got


def work(c):
    if c["op"] == "plan":
        ctx, new = _lengths(c)
        B, T = c["reqs"], sum(new) + c["slack"]
        fresh = sum(_pages(a + n, c["page"]) - _pages(a, c["page"]) for a, n in zip(ctx, new))
        # lengths in, per-request results out, per-token results out, one stack read and table write per fresh page, and the
        # table entry of the page each request was in the middle of
        return {"bytes": 4 * (3 * B + 3 * B + 2 * T + 2 * fresh + B), "flops": 0}
    if c["op"] in ("rope", "append"):
        T, H, Hkv, D = c["tokens"], c["heads"], c["kv_heads"], c["dim"]
        size = 2 if c["dtype"] == "bf16" else 4
        if c["op"] == "rope":
            return {"bytes": T * ((H + Hkv) * D * 2 * size + 4), "flops": T * (H + Hkv) * c["rotary"] * 3}
        return {"bytes": T * ((H + 2 * Hkv) * D * (size + 2) + 8), "flops": T * (H + Hkv) * c["rotary"] * 3}
    H, Hkv, D = c["heads"], c["kv_heads"], c["dim"]
    seen = _visible(c)
    T = sum(_lengths(c)[1])
    return {"bytes": sum(k for k, _ in seen) * Hkv * D * 4 + T * H * (D * 4 + 4),
            "flops": 4 * D * H * sum(p for _, p in seen)}


# ------------------------------------------------------------------------------------------------------------- exact
def exact(c, seed):
    if c["op"] == "plan":
        return None                          # whole numbers: there is nothing to round
    if c["op"] in ("rope", "append"):
        q, k, v, pos, table = _rope_inputs(c, seed)
        # the table's own values, as fractions of a turn; the product's whole turns drop out
        turns = torch.tensor([(w % _TWO64) / _TWO64 for w in table.tolist()], dtype=torch.float64, device=DEV)
        part = torch.remainder(pos.double()[:, None] * turns[None], 1.0)
        spin = torch.polar(torch.ones_like(part), 2.0 * math.pi * part)[:, None]
        if c.get("inverse"):
            spin = spin.conj()
        R = c["rotary"]

        def turn(x):
            y = x.double().clone()
            if c["layout"] == "half":
                z = torch.complex(y[..., :R // 2], y[..., R // 2:R]) * spin
                y[..., :R // 2], y[..., R // 2:R] = z.real, z.imag
            else:
                z = torch.complex(y[..., 0:R:2].contiguous(), y[..., 1:R:2].contiguous()) * spin
                y[..., 0:R:2], y[..., 1:R:2] = z.real, z.imag
            return y

        if c["op"] == "rope":
            return dict(q=turn(q), k=turn(k))
        s = prepare(c, seed)
        ck, cv = s["ck"].double(), s["cv"].double()
        at = s["slots"].long()
        ck[at // c["page"], at % c["page"]] = turn(k)
        cv[at // c["page"], at % c["page"]] = v.double()
        return dict(q=turn(q), k=ck, v=cv)
    s = _cache_inputs(c, seed)
    T, H, D = s["q"].shape
    out = torch.zeros(T, H, D, dtype=torch.float64, device=DEV)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=DEV)
    group, first = c["heads"] // c["kv_heads"], 0
    for b, (n, total) in enumerate(zip(s["new"], s["total"])):
        ids = s["table"][b, :_pages(total, c["page"])].long()
        key_pos = torch.arange(total, device=DEV)
        q_pos = torch.arange(total - n, total, device=DEV)
        hide = key_pos[None] > q_pos[:, None]
        if c["window"]:
            hide |= key_pos[None] <= q_pos[:, None] - c["window"]
        for kh in range(c["kv_heads"]):
            keys = s["k"][ids, :, kh].reshape(-1, D)[:total].double()
            vals = s["v"][ids, :, kh].reshape(-1, D)[:total].double()
            mine = slice(kh * group, (kh + 1) * group)
            z = torch.einsum("tgd,jd->gtj", s["q"][first:first + n, mine].double(), keys) / math.sqrt(D)
            z.masked_fill_(hide, -math.inf)
            out[first:first + n, mine] = (torch.softmax(z, -1) @ vals).transpose(0, 1)
            lse[first:first + n, mine] = torch.logsumexp(z, -1).T
        first += n
    return dict(out=out, lse=lse)
