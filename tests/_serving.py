"""Plain 64-bit forms of the serving operators and the bounds their GPU results are held to.

Bounds (derived from the arithmetic the header promises, before any run):
  rotation   angle: the fp32 value of the angle is within 2^-25 of a half turn (pi 2^-25 rad), sine and cosine within
             2 ulp of 1 (2^-22), two products and a sum of one rounding each (3 * 2^-24), amplitude 2^-24 more: together below
             6e-7 * amplitude * (|a| + |b|).  bf16 results add half an ulp, 2^-8 |value|.
  attention  scores: fp32 sums of D products, each rounding at most 2^-23 (also where the tensor cores truncate):
             e = D * 2^-23 * scale * max_j sum_d |q_d k_jd|, plus 2^-21 for the exponential and the scaling of its argument
             by log2(e) (|s - max| up to 16: beyond that a weight is below 2^-23 of the sum: 16 * 2^-24 * 2 < 2^-18).
             weights are rounded to bf16: 2^-8 each.  With A = sum_j w_j |v_j| / sum_j w_j an output element is within
             (2^-8 + 2 (e + 2^-18)) A of the exact one, plus its own rounding, 2^-8 |value|.
             lse: e + 2^-18 + 2^-23 |lse|.
"""
import math

import torch

DEV = "cuda"


def ref_rope(x, pos, freq_turns, rotary, pairs, inverse=False, amplitude=1.0):
    """x [T][H][D] (any float type) -> float64.  freq_turns: python floats, turns per position."""
    x = x.double()
    f = torch.tensor(freq_turns, dtype=torch.float64, device=x.device)
    ang = 2 * math.pi * torch.remainder(pos.double()[:, None] * f[None], 1.0)[:, None]
    c, s = torch.cos(ang) * amplitude, torch.sin(ang) * amplitude * (-1 if inverse else 1)
    y = x.clone()
    ia = torch.arange(0, rotary, 2) if pairs else torch.arange(rotary // 2)
    ib = ia + 1 if pairs else ia + rotary // 2
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    bound = torch.zeros_like(x)
    mag = (a.abs() + b.abs()) * abs(amplitude) * 6e-7
    bound[..., ia] = mag
    bound[..., ib] = mag
    return y, bound


def table_turns(table):
    return [(v % (1 << 64)) / float(1 << 64) for v in table.tolist()]


def within(got, ref, bound, what=""):
    got = got.double()
    assert got.shape == ref.shape, what
    bad = ~((got - ref).abs() <= bound)
    same = (got.isnan() & ref.isnan()) | (got == ref)      # NaN where the definition has NaN, equal infinities
    bad &= ~same
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} outside; first at "
                                 f"{bad.nonzero()[0].tolist()}: {got[tuple(bad.nonzero()[0])]} for {ref[tuple(bad.nonzero()[0])]} "
                                 f"+- {bound[tuple(bad.nonzero()[0])]}")


def ref_attention(q, k_req, v_req, new, kv, scale, causal=True, window=0):
    """q [T][H][D]; k_req[b], v_req[b]: [kv[b]][Hkv][D] of each request.  Returns (out, out bound, lse, lse bound), float64.
    Keys that a row does not see do not enter its sums at all."""
    T, H, D = q.shape
    dev = q.device
    out = torch.zeros(T, H, D, dtype=torch.float64, device=dev)
    bound = torch.zeros_like(out)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=dev)
    lb = torch.zeros_like(lse)
    t = 0
    for b, (n, L) in enumerate(zip(new, kv)):
        if n == 0 or L == 0:
            t += n
            continue
        G = H // k_req[b].shape[1]
        K = k_req[b].double().repeat_interleave(G, 1)
        V = v_req[b].double().repeat_interleave(G, 1)
        Q = q[t:t + n].double()
        S = torch.einsum("nhd,jhd->hnj", Q, K) * scale
        mag = torch.einsum("nhd,jhd->hnj", Q.abs(), K.abs()) * abs(scale)
        p = torch.arange(L - n, L, device=dev)[:, None]
        j = torch.arange(L, device=dev)[None]
        seen = torch.ones(n, L, dtype=torch.bool, device=dev)
        if causal:
            seen &= j <= p
        if window:
            seen &= j > p - window
        S = torch.where(seen, S, torch.full_like(S, -math.inf))
        mag = torch.where(seen, mag, torch.zeros_like(mag))
        m = S.amax(-1, keepdim=True)
        m = torch.where(torch.isneginf(m), torch.zeros_like(m), m)
        w = torch.exp(S - m)
        tot = w.sum(-1, keepdim=True)
        some = tot > 0
        # 0 * inf must not arise from keys that are not seen: their values are taken out row by row where needed
        fin = torch.isfinite(V)
        o = torch.einsum("hnj,jhd->hnd", w, torch.where(fin, V, torch.zeros_like(V)))
        A = torch.einsum("hnj,jhd->hnd", w, torch.where(fin, V, torch.zeros_like(V)).abs())
        if not bool(fin.all()):
            for jj in (~fin).any(-1).any(-1).nonzero().flatten().tolist():
                for i in range(n):
                    if bool(seen[i, jj]):
                        add = torch.where(fin[jj], torch.zeros_like(V[jj]), V[jj])
                        o[:, i] += add
        o = torch.where(some | tot.isnan(), o / tot, torch.zeros_like(o))
        A = torch.where(some, A / tot, torch.zeros_like(A))
        e = D * 2.0 ** -23 * mag.amax(-1, keepdim=True) + 2.0 ** -18
        e = torch.nan_to_num(e, nan=0.0, posinf=0.0)
        out[t:t + n] = o.permute(1, 0, 2)
        bound[t:t + n] = ((2.0 ** -8 + 2 * e) * A + 2.0 ** -8 * o.abs().nan_to_num(posinf=0.0)).permute(1, 0, 2)
        ls = torch.log(tot) + m
        lse[t:t + n] = ls.squeeze(-1).T
        lb[t:t + n] = (e + 2.0 ** -23 * ls.abs().nan_to_num(posinf=0.0)).squeeze(-1).T
        t += n
    return out, bound, lse, lb


def make_cache(gen, kv, page, Hkv, D, order="nhd", fill=float("nan"), spare=3, std=1.0):
    """Random keys and values of each request, scattered over the pages of a cache whose other entries hold `fill`.
    Returns (k, v cache views [pages][page][Hkv][D], block table, per-request keys, values)."""
    need = [-(-n // page) for n in kv]
    n_pages = sum(need) + spare
    shape = (n_pages, page, Hkv, D) if order == "nhd" else (n_pages, Hkv, page, D)
    ck = torch.full(shape, fill, dtype=torch.bfloat16, device=DEV)
    cv = torch.full(shape, fill, dtype=torch.bfloat16, device=DEV)
    if order == "hnd":
        ck, cv = ck.permute(0, 2, 1, 3), cv.permute(0, 2, 1, 3)
    perm = torch.randperm(n_pages, generator=gen, device=DEV)
    width = max(max(need), 1) + 1
    table = torch.full((len(kv), width), -1, dtype=torch.int32, device=DEV)
    ks, vs, at = [], [], 0
    for b, n in enumerate(kv):
        ids = perm[at:at + need[b]]
        at += need[b]
        table[b, :need[b]] = ids.to(torch.int32)
        k = (torch.randn(n, Hkv, D, generator=gen, device=DEV) * std).to(torch.bfloat16)
        v = torch.randn(n, Hkv, D, generator=gen, device=DEV).to(torch.bfloat16)
        j = torch.arange(n, device=DEV)
        if n:
            ck[ids[j // page], j % page] = k
            cv[ids[j // page], j % page] = v
        ks.append(k)
        vs.append(v)
    return ck, cv, table, ks, vs


def offsets(new):
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device=DEV)
