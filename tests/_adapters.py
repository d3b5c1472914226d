"""Plain 64-bit forms of the calls for many adapters and of the AdamW step, and the bounds their GPU results are held to.

Bounds (derived from the arithmetic the header promises, before any run):
  adapters   x', x' A (and dv, du) are carried as pairs of bf16 numbers: what is left after the first is at most 2^-8 of the value
             (half a step of 2^-7), of that after the second again 2^-8: 2^-16 of the value at worst, and the product of the two
             seconds, left out where both sides are pairs, 2^-16 as well.  Sums are fp32, each addition off by at most 2^-23 of the
             terms' absolute sum (also where the tensor cores truncate).  With Abs = the same products of absolute values, K the
             terms of all sums an output goes through, c the pairs it goes through:
                 |error| <= (c 2^-16 + (K + 8) 2^-23) Abs  +  half a step of the result
             Over a whole output the errors of different terms are independent and the pairs' are evenly spread over their range, a
             third of the worst case and less: the 2-norm of the error is below c 2^-17 + 2^-19 of the result's 2-norm.  (One bf16
             number in place of a pair would have 2^-10 there.)
  AdamW      every step of the formulas in fp32, about ten roundings of 2^-24 and two approximate divisions of 2^-22: 2^-20 of
             |update| + |p|; the averages three roundings, 2^-22 of their terms' absolute sum.
"""
import torch

DEV = "cuda"


def requests(lengths, ids, tokens=None):
    """cu, ids as the calls take them, and the buffers' rows."""
    cu = [0]
    for n in lengths:
        cu.append(cu[-1] + n)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    return i32(cu), i32(ids), tokens if tokens is not None else max(cu[-1], 1)


def ref_plan(cu, ids, n, tokens):
    """rows, start as lists."""
    mine = [[] for _ in range(n)]
    for b, a in enumerate(ids):
        if 0 <= a < n:
            mine[a] += range(cu[b], cu[b + 1])
    start = [0]
    for m in mine:
        start.append(start[-1] + len(m))
    rows = [t for m in mine for t in m]
    return rows + [-1] * (tokens - len(rows)), start


def make_bank(qb, n, d_in, d_out, l1, l2, r, ranks=None, seed=0, gain=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    P, Q = d_in // l1, d_out // l2
    A = (torch.randn(n, P, r, generator=g, device=DEV) * (2 * gain / P ** 0.5)).bfloat16()
    B = (torch.randn(n, r, Q, generator=g, device=DEV) * (gain / r ** 0.5)).bfloat16()
    s = torch.rand(n, generator=g, device=DEV) + 0.5
    rk = None
    if ranks is not None:
        rk = torch.tensor(ranks, dtype=torch.int32, device=DEV)
        keep = torch.arange(r, device=DEV) < rk[:, None]
        A, B = A * keep[:, None], B * keep[:, :, None]
    return qb.AdapterBank(d_in, d_out, l1, l2, A.contiguous(), B.contiguous(), s, rk)


def _wide(bank, a):
    return bank.A[a].double(), bank.B[a].double(), float(bank.scaling[a])


def ref_fwd(bank, cu, ids, X, Y):
    """(Y', Abs): what the call leaves in Y, and the absolute sums behind each element."""
    Y, bound = Y.double(), torch.zeros_like(Y, dtype=torch.float64)
    for b, a in enumerate(ids):
        t = slice(cu[b], cu[b + 1])
        if a < 0 or cu[b] == cu[b + 1]:
            continue
        A, B, s = _wide(bank, a)
        x = X[t].double().view(-1, A.shape[0], bank.lambda_in)
        Y[t] += (x.mean(-1) @ A @ B * s).repeat_interleave(bank.lambda_out, 1)
        bound[t] = (x.abs().mean(-1) @ A.abs() @ B.abs() * s).repeat_interleave(bank.lambda_out, 1)
    return Y, bound


def ref_bwd(bank, cu, ids, X, dY, dX):
    """(dX', dA, dB) and their Abs."""
    out = [dX.double(), torch.zeros_like(bank.A, dtype=torch.float64), torch.zeros_like(bank.B, dtype=torch.float64)]
    bound = [torch.zeros_like(x) for x in out]
    for b, a in enumerate(ids):
        t = slice(cu[b], cu[b + 1])
        if a < 0 or cu[b] == cu[b + 1]:
            continue
        A, B, s = _wide(bank, a)
        x = X[t].double().view(-1, A.shape[0], bank.lambda_in)
        y = dY[t].double().view(-1, B.shape[1], bank.lambda_out) * s
        for to, f in ((out, lambda z: z), (bound, torch.abs)):
            xp, dv, fa, fb = f(x).mean(-1), f(y).sum(-1), f(A), f(B)
            du = dv @ fb.T
            to[0][t] += (du @ fa.T / bank.lambda_in).repeat_interleave(bank.lambda_in, 1)
            to[1][a] += xp.T @ du
            to[2][a] += (xp @ fa).T @ dv
    return out, bound


def check(got, want, bound, pairs, terms, what, base=None):
    """The element bound and, where there is enough to average over, the bound of the 2-norm.  `base`: what was there before,
    whose part of the 2-norm says nothing."""
    got = got.double()
    assert torch.isfinite(got).all(), what
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[what[1]]
    err = (got - want).abs()
    limit = (pairs * 2.0 ** -16 + (terms + 8) * 2.0 ** -23) * bound + half * want.abs() + 1e-30
    worst = float((err / limit).max())
    assert worst <= 1.0, (what, worst)
    if what[1] is torch.float32 and want.numel() >= 4096:
        size = (want - base.double() if base is not None else want).norm()
        off = err - 2.0 ** -24 * want.abs()            # the rounding of the sum itself is no part of it
        assert float(off.clamp(min=0).norm()) <= (pairs * 2.0 ** -17 + 2.0 ** -19) * float(size), what
