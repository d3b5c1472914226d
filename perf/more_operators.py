"""Performance cases of the operators around many adapters over one frozen base weight: rows sorted by adapter, the
adapters of many requests beside a shared projection with their gradients, and the AdamW step over all of them.

``listed()`` and ``draw(rng)`` give cases, ``prepare(case, seed)`` the tensors a caller holds before a call,
``run(state)`` one call: with ``own`` set through the library's entry points, otherwise in elementary torch operations
in 32 bits, rounded once at the end.  ``exact(case, seed)`` computes the same outputs from the definitions in 64 bits.

Notation: R requests with the rows cu[b] .. cu[b + 1] - 1 of X and Y; request b uses adapter ids[b] of n, or none (-1).
Adapter a is A[a] [P][r], B[a] [r][Q] with P = d_in / lambda_in, Q = d_out / lambda_out and the factor s[a].
"""
import math
import random

import torch

own = False
DEV = "cuda"
BLOCK = 256                                  # elements that share a scale where the optimizer's states are held in 8 bits
_M32 = 0xffffffff


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    wide = dict(lambda_in=64, lambda_out=8)              # the geometry of the mergeable adapters
    four = dict(lambda_in=4, lambda_out=4)               # one balancing factor on both sides
    return [
        # one step of a server: 48 requests decode, 16 adapters, a few requests without any; latency is all that counts
        dict(name="plan decode 48", op="plan", reqs=48, adapters=16, long=0, long_rows=0, none=5, slack=0, lens=1),
        # a large mixed step: 700 requests, 24 of them bring prompt chunks, unused rows behind them
        dict(name="plan mixed 700", op="plan", reqs=700, adapters=100, long=24, long_rows=811, none=60, slack=331, lens=2),
        # a lone user decoding beside the 4096 x 4096 projection
        dict(name="fwd 1 token", op="fwd", reqs=1, adapters=8, long=0, long_rows=0, none=0, slack=0, lens=3, d_in=4096,
             d_out=4096, rank=256, uneven=False, dtype="bf16", **wide),
        # a busy server: 48 requests share 16 adapters of rank 64
        dict(name="fwd decode 48 of 16", op="fwd", reqs=48, adapters=16, long=0, long_rows=0, none=3, slack=0, lens=4,
             d_in=4096, d_out=11008, rank=64, uneven=False, dtype="bf16", **four),
        # every request its own adapter: bound by reading them
        dict(name="fwd decode 200 of 200", op="fwd", reqs=200, adapters=200, long=0, long_rows=0, none=0, slack=0, lens=5,
             d_in=5120, d_out=5120, rank=256, uneven=False, dtype="bf16", **four),
        # a step that mixes decoding requests with two prompt chunks; adapters of uneven rank, unused rows
        dict(name="fwd mixed 32", op="fwd", reqs=32, adapters=12, long=2, long_rows=1021, none=4, slack=19, lens=6,
             d_in=5120, d_out=13824, rank=256, uneven=True, dtype="bf16", **wide),
        # a training batch of four adapters, about 7000 rows in sequences of up to 512
        dict(name="fwd train 7k of 4", op="fwd", reqs=16, adapters=4, long=16, long_rows=512, none=0, slack=0, lens=7,
             d_in=4096, d_out=11008, rank=256, uneven=False, dtype="bf16", **four),
        # gradients of a small training batch, three adapters
        dict(name="bwd 1800 of 3", op="bwd", reqs=5, adapters=3, long=5, long_rows=409, none=0, slack=3, lens=8, d_in=4096,
             d_out=4096, rank=256, uneven=False, dtype="bf16", **four),
        # gradients of a large one beside the widest projection, uneven sequences, input gradient in 32 bits
        dict(name="bwd 6700 of 6", op="bwd", reqs=13, adapters=6, long=13, long_rows=630, none=1, slack=1, lens=9, d_in=13824,
             d_out=5120, rank=256, uneven=True, dtype="f32", **wide),
        # the optimizer step of one small linear's adapter, clipped: latency
        dict(name="step one linear", op="step", layers=1, linears="4096x4096", rank=256, bits=32, grad="f32", clip=True,
             odd=0, steps=0, **wide),
        # all adapters of a 13B-shaped model (40 layers of seven linears), states in 32 bits
        dict(name="step 40 layers 32 bits", op="step", layers=40, linears="5120x5120 " * 4 + "13824x5120 " * 2 + "5120x13824",
             rank=128, bits=32, grad="f32", clip=False, odd=0, steps=100, **four),
        # the same with states in 8 bits and gradients in 16, clipped by their global norm
        dict(name="step 40 layers 8 bits", op="step", layers=40, linears="5120x5120 " * 4 + "13824x5120 " * 2 + "5120x13824",
             rank=128, bits=8, grad="bf16", clip=True, odd=0, steps=1000, **four),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["plan", "fwd", "fwd", "fwd", "bwd", "bwd", "step", "step"])
    lens = rng.randrange(1 << 30)
    lam = rng.choice([(64, 8), (4, 4), (4, 4), (8, 8), (2, 4), (1, 1), (16, 2)])
    geo = dict(lambda_in=lam[0], lambda_out=lam[1])
    if op == "plan":
        reqs = _log_int(rng, 8, 700)
        long = min(reqs, rng.randrange(24))
        return dict(op=op, reqs=reqs, adapters=_log_int(rng, 5, 200), long=long, long_rows=_log_int(rng, 2, 800),
                    none=rng.randrange(1 + reqs // 4), slack=rng.randrange(300), lens=lens)
    if op == "step":
        # between one linear and a seventh of the largest listed model; some tensors of odd sizes
        return dict(op=op, layers=_log_int(rng, 1, 40), linears=rng.choice(["4096x4096", "11008x4096", "5120x5120 13824x5120", "1024x1024"]),
                    rank=rng.choice([8, 16, 64, 64, 128]), bits=rng.choice([8, 32]), grad=rng.choice(["f32", "bf16"]),
                    clip=rng.random() < 0.5, odd=rng.choice([0, 0, 1, 77]), steps=_log_int(rng, 1, 5000) - 1, **geo)
    d_in, d_out = rng.choice([1024, 4096, 4096, 5120, 11008]), rng.choice([1024, 4096, 4096, 5120, 11008])
    rank = rng.choice([8, 16, 32, 64, 64, 128, 256])
    kind = rng.choice(["decode", "decode", "mixed", "train"]) if op == "fwd" else "train"
    reqs = {"decode": _log_int(rng, 1, 200), "mixed": _log_int(rng, 2, 64), "train": _log_int(rng, 1, 12)}[kind]
    long = {"decode": 0, "mixed": rng.choice([1, 2]), "train": reqs}[kind]
    rows = _log_int(rng, 20, 1000) if long else 0
    if kind == "train":
        rows = max(1, min(rows, 5000 // reqs))
    # bank of at most 300 MB, and (padded to the longest adapter's rows) at most 12000 rows
    adapters = _log_int(rng, 1, max(1, min(reqs + 3, int(3e8 / (2 * rank * (d_in // lam[0] + d_out // lam[1]))),
                                           12000 // (max(1, long) * max(1, rows)) if long else 200)))
    return dict(op=op, reqs=reqs, adapters=adapters, long=long, long_rows=rows, none=rng.randrange(1 + reqs // 8),
                slack=rng.choice([0, 0, 1, 13]), lens=lens, d_in=d_in, d_out=d_out, rank=rank, uneven=rng.random() < 0.3,
                dtype=rng.choice(["bf16", "bf16", "f32"]), **geo)


# ------------------------------------------------------------------------------------------------------------ inputs
def _requests(c):
    """(rows, adapter) of each request: a property of the case, equal for all seeds.  `long` requests bring up to long_rows
    rows, the others one; `none` of them have no adapter."""
    r = random.Random(c["lens"])
    new = [1] * c["reqs"]
    for b in range(c["long"]):
        new[b] = c["long_rows"] if b % 2 == 0 else r.randint(1 + c["long_rows"] // 2, c["long_rows"])
    ids = [b if c["adapters"] >= c["reqs"] else r.randrange(c["adapters"]) for b in range(c["reqs"])]
    r.shuffle(ids)
    for b in r.sample(range(c["reqs"]), min(c["none"], c["reqs"] - 1)):
        ids[b] = -1
    order = list(range(c["reqs"]))
    r.shuffle(order)
    return [new[b] for b in order], [ids[b] for b in order]


def _rows_of(c):
    """Rows of each adapter."""
    new, ids = _requests(c)
    got = [0] * c["adapters"]
    for n, a in zip(new, ids):
        if a >= 0:
            got[a] += n
    return got


def _ranks(c):
    """Rank of each adapter, before they are dealt out."""
    r = random.Random(c["lens"] + 1)
    return [r.choice([k for k in (8, 16, 64, 256, c["rank"]) if k <= c["rank"]]) if c["uneven"] else c["rank"]
            for _ in range(c["adapters"])]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + 29)


def _randn(g, *shape, dtype=torch.bfloat16, gain=1.0):
    """Normal values of the given type, drawn in pieces so that no 32-bit copy of a large tensor exists."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    for piece in out.view(-1).split(1 << 26):
        piece.copy_(torch.randn(piece.shape, generator=g, device=DEV) * gain)
    return out


def _plan_inputs(c, seed):
    """Offsets and adapters; another seed brings the requests in another order and deals out other adapters."""
    new, ids = _requests(c)
    order = list(range(len(new)))
    random.Random(seed).shuffle(order)
    new, ids = [new[b] for b in order], [ids[b] for b in order]
    perm = torch.randperm(c["adapters"], generator=_generator(seed), device=DEV).to(torch.int32)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    ids = _i32(ids)
    return dict(cu=_i32(cu), ids=torch.where(ids >= 0, perm[ids.clamp(min=0).long()], ids), tokens=cu[-1] + c["slack"],
                slot=perm.long())


def _sorted_rows(s, n):
    """rows and start of the plan, in torch operations."""
    tokens = s["tokens"]
    at = torch.arange(tokens, device=DEV)
    b = torch.searchsorted(s["cu"][1:].long(), at, right=True)
    key = torch.where(b < len(s["ids"]), s["ids"][b.clamp(max=len(s["ids"]) - 1)].long(), -1)
    key = torch.where(key < 0, n, key)
    order = torch.argsort(key, stable=True)
    start = torch.searchsorted(key[order].contiguous(), torch.arange(n + 1, device=DEV))
    rows = torch.where(at < start[n], order, -1)
    return rows.to(torch.int32), start.to(torch.int32)


def _adapter_inputs(c, seed):
    s = _plan_inputs(c, seed)
    n, r, T = c["adapters"], c["rank"], s["tokens"]
    P, Q = c["d_in"] // c["lambda_in"], c["d_out"] // c["lambda_out"]
    s["rows"], s["start"] = _sorted_rows(s, n)
    g = _generator(seed + 1)
    # trained adapters: what they add is about as large as what is there
    s["A"], s["B"] = _randn(g, n, P, r, gain=2.0 / math.sqrt(P)), _randn(g, n, r, Q, gain=1.0 / math.sqrt(r))
    s["scaling"] = torch.rand(n, generator=g, device=DEV) + 0.5
    s["ranks"] = None
    if c["uneven"]:                          # adapters of a lower rank have zeros behind it
        s["ranks"] = torch.empty(n, dtype=torch.int32, device=DEV)
        s["ranks"][s["slot"]] = _i32(_ranks(c))
        keep = torch.arange(r, device=DEV) < s["ranks"][:, None]
        s["A"].mul_(keep[:, None, :])
        s["B"].mul_(keep[:, :, None])
    dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    s["X"] = _randn(g, T, c["d_in"])
    if c["op"] == "fwd":
        s["Y"] = _randn(g, T, c["d_out"], dtype=dtype)                # what the shared projection has written
    else:
        s["dY"] = _randn(g, T, c["d_out"])
        s["dX"] = _randn(g, T, c["d_in"], dtype=dtype)                # what the shared projection's backward pass has written
    return s


def _tensor_sizes(c):
    """Elements of each trained tensor: A and B of every linear of every layer, some with `odd` elements more."""
    got = []
    for k in range(c["layers"]):
        for j, lin in enumerate(c["linears"].split()):
            o, i = (int(v) for v in lin.split("x"))
            extra = c["odd"] if (k + j) % 3 == 0 else 0
            got += [i // c["lambda_in"] * c["rank"] + extra, o // c["lambda_out"] * c["rank"]]
    return got


def _step_inputs(c, seed):
    """One buffer per role; tensor k is the elements at[k] .. at[k] + size[k] of it, every tensor begins a new block."""
    sizes, at, total = _tensor_sizes(c), [], 0
    for n in sizes:
        at.append(total)
        total += -(-n // BLOCK) * BLOCK
    g = _generator(seed)
    blocks = total // BLOCK
    used = torch.zeros(total, dtype=torch.bool, device=DEV)
    for a, n in zip(at, sizes):
        used[a:a + n] = True
    # gradients of very uneven size over the blocks, averages as after some steps on such gradients
    size = torch.exp(torch.randn(blocks, 1, generator=g, device=DEV)) * 1e-3
    grad = (torch.randn(blocks, BLOCK, generator=g, device=DEV) * size).view(-1) * used
    started = 0.0 if c["steps"] == 0 else 1.0
    m = (torch.randn(blocks, BLOCK, generator=g, device=DEV) * size * 0.3 * started).view(-1) * used
    root = ((0.7 + 0.6 * torch.rand(blocks, BLOCK, generator=g, device=DEV)) * size * started).view(-1) * used
    s = dict(sizes=sizes, at=at, p=_randn(g, total, dtype=torch.float32, gain=0.02) * used,
             grad=grad if c["grad"] == "f32" else grad.to(torch.bfloat16),
             copy=torch.zeros(total, dtype=torch.bfloat16, device=DEV), steps=_i32([c["steps"]]),
             lr=torch.tensor([2e-4], dtype=torch.float32, device=DEV))
    if c["bits"] == 32:
        s["m"], s["v"] = m, root * root
    else:
        for name, x in (("m", m), ("v", root)):              # the second average is held by its square root
            scale = x.view(-1, BLOCK).abs().amax(-1, keepdim=True) / 448.0
            s[name + "_scale"] = scale.view(-1)
            s[name] = (x.view(-1, BLOCK) / torch.where(scale > 0, scale, 1.0)).to(torch.float8_e4m3fn).view(-1)
    return s


_HYPER = dict(betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, seed=17)


def _max_norm(c):
    return 0.3 if c["clip"] else 0.0


def prepare(case, seed):
    s = dict(case=case, scratch={})              # scratch: the workspace or handle that a caller keeps between its calls
    if case["op"] == "plan":
        s.update(_plan_inputs(case, seed))
        s["rows"], s["start"] = (torch.empty(k, dtype=torch.int32, device=DEV) for k in (s["tokens"], case["adapters"] + 1))
    elif case["op"] == "step":
        s.update(_step_inputs(case, seed))
    else:
        s.update(_adapter_inputs(case, seed))
        if case["op"] == "bwd":
            s["dA"], s["dB"] = (torch.empty(s[k].shape, dtype=torch.float32, device=DEV) for k in "AB")
    return s


# --------------------------------------------------------------------------------------------------------------- run
def run(s):
    return (_run_own if own else _run_plain)[s["case"]["op"]](s)


def _own_plan(s):
    from paper_2407_17029_b200 import binding as qb
    p = qb.adapter_plan(s["cu"], s["ids"], s["case"]["adapters"], s["tokens"], outs=(s["rows"], s["start"]))
    return dict(rows=p.rows, start=p.start)


def _own_bank(s, qb):
    c = s["case"]
    return qb.AdapterBank(c["d_in"], c["d_out"], c["lambda_in"], c["lambda_out"], s["A"], s["B"], s["scaling"], s["ranks"])


def _own_fwd(s):
    from paper_2407_17029_b200 import binding as qb
    bank = _own_bank(s, qb)
    if "ws" not in s["scratch"]:
        s["scratch"]["ws"] = qb.alloc_adapters_workspace(bank, s["tokens"])
    return dict(Y=qb.adapters_fwd(bank, qb.AdapterPlan(s["rows"], s["start"]), s["X"], s["Y"], ws=s["scratch"]["ws"]))


def _own_bwd(s):
    from paper_2407_17029_b200 import binding as qb
    bank = _own_bank(s, qb)
    if "ws" not in s["scratch"]:
        s["scratch"]["ws"] = qb.alloc_adapters_workspace(bank, s["tokens"], backward=True)
    dX, dA, dB = qb.adapters_bwd(bank, qb.AdapterPlan(s["rows"], s["start"]), s["X"], s["dY"], s["dX"], outs=(s["dA"], s["dB"]),
                                 ws=s["scratch"]["ws"])
    return dict(dX=dX, dA=dA, dB=dB)


def _own_step(s):
    from paper_2407_17029_b200 import binding as qb
    c = s["case"]
    if "opt" not in s["scratch"]:
        part = lambda x: [x[a:a + n] for a, n in zip(s["at"], s["sizes"])]  # noqa: E731
        scales = lambda x: [x[a // BLOCK:a // BLOCK + -(-n // BLOCK)] for a, n in zip(s["at"], s["sizes"])]  # noqa: E731
        states = dict(m=part(s["m"]), v=part(s["v"]))
        if c["bits"] == 8:
            states.update(m_scale=scales(s["m_scale"]), v_scale=scales(s["v_scale"]))
        s["scratch"]["opt"] = qb.AdamW(part(s["p"]), part(s["grad"]), copies=part(s["copy"]), state_bits=c["bits"], states=states,
                                       lr=s["lr"], steps=s["steps"], max_norm=_max_norm(c), **_HYPER)
    s["scratch"]["opt"].step()
    return _step_outputs(s)


def _step_outputs(s):
    """Parameters, their 16-bit copy, the states; states in 8 bits as the numbers of their 8-bit type beside their scales."""
    return {k: s[k] for k in ("p", "copy", "m", "v", "m_scale", "v_scale", "steps") if k in s}


def _plain_plan(s):
    rows, start = _sorted_rows(s, s["case"]["adapters"])
    s["rows"].copy_(rows)
    s["start"].copy_(start)
    return dict(rows=s["rows"], start=s["start"])


def _padded(s):
    """Rows of each adapter, padded to the longest: row numbers [n][N] and which of them are there."""
    N = max(1, max(_rows_of(s["case"])))
    at = s["start"][:-1, None].long() + torch.arange(N, device=DEV)
    real = at < s["start"][1:, None]
    return torch.where(real, s["rows"][at.clamp(max=len(s["rows"]) - 1)], 0).long(), real


def _plain_fwd(s):
    c = s["case"]
    P, Q = c["d_in"] // c["lambda_in"], c["d_out"] // c["lambda_out"]
    at, real = _padded(s)
    x = s["X"][at].to(torch.float32).view(*at.shape, P, c["lambda_in"]).mean(-1)
    v = (x @ s["A"].to(torch.float32)) @ s["B"].to(torch.float32) * s["scaling"][:, None, None]
    at, v = at[real], v[real]
    y = s["Y"][at].to(torch.float32).view(-1, Q, c["lambda_out"]) + v[..., None]
    s["Y"][at] = y.view(-1, c["d_out"]).to(s["Y"].dtype)
    return dict(Y=s["Y"])


def _plain_bwd(s):
    c = s["case"]
    P, Q = c["d_in"] // c["lambda_in"], c["d_out"] // c["lambda_out"]
    at, real = _padded(s)
    A, B = s["A"].to(torch.float32), s["B"].to(torch.float32)
    x = s["X"][at].to(torch.float32).view(*at.shape, P, c["lambda_in"]).mean(-1)
    dv = s["dY"][at].to(torch.float32).view(*at.shape, Q, c["lambda_out"]).sum(-1) * s["scaling"][:, None, None]
    x, dv = x * real[..., None], dv * real[..., None]
    du = dv @ B.transpose(1, 2)
    s["dA"].copy_(x.transpose(1, 2) @ du)
    s["dB"].copy_((x @ A).transpose(1, 2) @ dv)
    dx = ((du @ A.transpose(1, 2)) / c["lambda_in"])[real]
    at = at[real]
    y = s["dX"][at].to(torch.float32).view(-1, P, c["lambda_in"]) + dx[..., None]
    s["dX"][at] = y.view(-1, c["d_in"]).to(s["dX"].dtype)
    return dict(dX=s["dX"], dA=s["dA"], dB=s["dB"])


def _mix(x):
    """32 bits that look random, of a number of 32 bits (held in 64)."""
    x = ((x ^ (x >> 16)) * 0xA3C59AC3) & _M32
    x = ((x ^ (x >> 15)) * 0x5D8E3B97) & _M32
    return x ^ (x >> 16)


def _to_8_bits(x, bits16):
    """Codes (e4m3) and scales of a state: |x| / scale is rounded down or up to a neighbour, up where the fraction that is
    lost and 16 random bits together make a whole."""
    x = x.view(-1, BLOCK)
    top = x.abs().amax(-1, keepdim=True)
    top = torch.where(top < 2.0 ** -118, torch.zeros_like(top), top)
    y = (x.abs() * torch.where(top > 0, 448.0 / top, torch.zeros_like(top))).clamp(max=448.0)
    bits16 = bits16.view(-1, BLOCK)
    normal = ((y.contiguous().view(torch.int32).long() + (bits16 << 4)) >> 20) - 960
    small = torch.floor(y * 512.0 + bits16.to(torch.float32) * 2.0 ** -16).long()
    code = torch.where(y >= 2.0 ** -6, normal, small) | ((x < 0).long() << 7)
    return code.to(torch.uint8).view(torch.float8_e4m3fn).view(-1), (top * (1.0 / 448.0)).view(-1)


def _plain_step(s):
    c = s["case"]
    (b1, b2), eps, wd = _HYPER["betas"], _HYPER["eps"], _HYPER["weight_decay"]
    g = s["grad"].to(torch.float32)
    if c["clip"]:
        norm = g.double().square().sum().sqrt()
        g = g * torch.where(norm > _max_norm(c), _max_norm(c) / norm, 1.0).to(torch.float32)
    s["steps"] += 1
    t = s["steps"].double()
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
        m.mul_(b1).add_(g, alpha=1 - b1)
        v.mul_(b2).add_(g * g, alpha=1 - b2)
    else:
        m = s["m"].to(torch.float32).view(-1, BLOCK) * s["m_scale"][:, None] * b1
        v = (s["v"].to(torch.float32).view(-1, BLOCK) * s["v_scale"][:, None]).square() * b2
        m, v = m.view(-1) + g * (1 - b1), v.view(-1) + g * g * (1 - b2)
    step = (m / (1 - b1 ** t).to(torch.float32)) / ((v / (1 - b2 ** t).to(torch.float32)).sqrt() + eps)
    s["p"].sub_(s["lr"] * (step + wd * s["p"]))
    s["copy"].copy_(s["p"])
    if c["bits"] == 8:
        key = _mix((_mix(s["steps"].long() * 0 + _HYPER["seed"]) + s["steps"].long()) & _M32)
        x = _mix((torch.arange(m.numel(), device=DEV) * 0x9E3779B1 + key) & _M32)
        for name, state, bits in (("m", m, x & 0xffff), ("v", v.sqrt(), x >> 16)):
            code, scale = _to_8_bits(state, bits)
            s[name].copy_(code)
            s[name + "_scale"].copy_(scale)
    return _step_outputs(s)


_run_own = dict(plan=_own_plan, fwd=_own_fwd, bwd=_own_bwd, step=_own_step)
_run_plain = dict(plan=_plain_plan, fwd=_plain_fwd, bwd=_plain_bwd, step=_plain_step)


# -------------------------------------------------------------------------------------------------------------- work
def work(c):
    if c["op"] == "plan":
        new, _ = _requests(c)
        return {"bytes": 4 * (2 * c["reqs"] + 1 + sum(new) + c["slack"] + c["adapters"] + 1), "flops": 0}
    if c["op"] == "step":
        n = sum(_tensor_sizes(c))
        grad = 4 if c["grad"] == "f32" else 2
        state = 16.0 if c["bits"] == 32 else 4.0 + 16.0 / BLOCK
        return {"bytes": n * (8 + 2 + grad + state), "flops": 15 * n}
    P, Q = c["d_in"] // c["lambda_in"], c["d_out"] // c["lambda_out"]
    size = 2 if c["dtype"] == "bf16" else 4
    rows, ranks = _rows_of(c), _ranks(c)
    T = sum(rows)
    bank = sum(2 * r * (P + Q) for k, r in zip(rows, ranks) if k)
    if c["op"] == "fwd":
        return {"bytes": T * (2 * c["d_in"] + 2 * size * c["d_out"]) + bank,
                "flops": sum(2 * k * r * (P + Q) for k, r in zip(rows, ranks))}
    return {"bytes": T * (2 * c["d_in"] + 2 * c["d_out"] + 2 * size * c["d_in"]) + bank + 4 * c["adapters"] * c["rank"] * (P + Q),
            "flops": sum(2 * k * r * (3 * P + 2 * Q) for k, r in zip(rows, ranks))}


# ------------------------------------------------------------------------------------------------------------- exact
def exact(c, seed):
    if c["op"] == "plan":
        return None                          # whole numbers: there is nothing to round
    if c["op"] == "step":
        return _exact_step(c, seed)
    s = _adapter_inputs(c, seed)
    n, l1, l2 = c["adapters"], c["lambda_in"], c["lambda_out"]
    new, ids = s["cu"].diff().tolist(), s["ids"].tolist()
    if c["op"] == "fwd":
        Y = s["Y"].double()
    else:
        dX = s["dX"].double()
        dA, dB = (torch.zeros(s[k].shape, dtype=torch.float64, device=DEV) for k in "AB")
    first = 0
    for rows, a in zip(new, ids):            # request by request, as the definition has it
        t = slice(first, first + rows)
        first += rows
        if a < 0:
            continue
        A, B, scale = s["A"][a].double(), s["B"][a].double(), float(s["scaling"][a])
        # the pooled input as a product with the matrix of means, the repeated output as its transpose's
        pooled = torch.nn.functional.avg_pool1d(s["X"][t].double()[:, None], l1)[:, 0]
        if c["op"] == "fwd":
            Y[t] += scale * torch.repeat_interleave(torch.linalg.multi_dot([pooled, A, B]) if rows > 1 else pooled @ A @ B, l2, 1)
            continue
        dv = torch.nn.functional.avg_pool1d(s["dY"][t].double()[:, None], l2)[:, 0] * (l2 * scale)
        du = torch.einsum("tq,rq->tr", dv, B)
        dX[t] += torch.repeat_interleave(torch.einsum("tr,pr->tp", du, A) / l1, l1, 1)
        dA[a] += torch.einsum("tp,tr->pr", pooled, du)
        dB[a] += torch.einsum("tr,tq->rq", pooled @ A, dv)
    return dict(Y=Y) if c["op"] == "fwd" else dict(dX=dX, dA=dA, dB=dB)


def _exact_step(c, seed):
    s = _step_inputs(c, seed)
    (b1, b2), eps, wd = _HYPER["betas"], _HYPER["eps"], _HYPER["weight_decay"]
    t, lr = c["steps"] + 1, float(s["lr"])
    factor = 1.0
    if c["clip"]:
        norm = math.sqrt(float(torch.dot(s["grad"].double(), s["grad"].double())))
        factor = min(1.0, _max_norm(c) / norm)
    g = s["grad"].double() * factor
    if c["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        wide = lambda k: s[k].to(torch.float64) * s[k + "_scale"].double().repeat_interleave(BLOCK)  # noqa: E731
        m, v = wide("m"), wide("v") ** 2
    m = torch.lerp(g, m, b1)
    v = torch.lerp(g * g, v, b2)
    del g
    hat = m / (1.0 - b1 ** t) / (torch.sqrt(v / (1.0 - b2 ** t)) + eps)
    p = s["p"].double() * (1.0 - lr * wd) - lr * hat
    if c["bits"] == 32:
        return dict(p=p, copy=p, m=m, v=v)
    # states in 8 bits have no single value: what is held is a neighbour of it
    return dict(p=p, copy=p, m_scale=m.view(-1, BLOCK).abs().amax(-1) / 448.0, v_scale=v.sqrt().view(-1, BLOCK).amax(-1) / 448.0)
