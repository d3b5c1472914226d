"""Rotary positions, the paged cache's plan and the attention over it, against plain forms in 64 bits (tests/_serving.py).
Unused cache entries hold NaN throughout, so a read past a request's keys shows in its results."""

import pytest
import torch

from tests._serving import DEV, make_cache, offsets, ref_attention, ref_rope, table_turns, within

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _qb():
    from paper_2407_17029_b200 import binding as qb
    return qb


# ------------------------------------------------------------------------------------------------------------- rotary
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,Hk,D,rot", [(1, 1, 1, 64, 64), (1, 32, 8, 128, 128), (7, 5, 5, 80, 32), (33, 3, 1, 128, 64),
                                          (5, 2, 2, 24, 10), (130, 40, 40, 128, 128), (3, 4, 1, 256, 192), (2, 1, 1, 2, 2)])
def test_rope_forward_and_inverse(pairs, dtype, T, H, Hk, D, rot):
    qb = _qb()
    g = _gen(T + H + D)
    q = torch.randn(T, H, D, generator=g, device=DEV).to(dtype)
    k = torch.randn(T, Hk, D, generator=g, device=DEV).to(dtype)
    pos = torch.randint(0, 1 << 20, (T,), generator=g, device=DEV).to(torch.int32)
    pos[0] = 0
    tab = qb.rope_table(rot)
    cfg = qb.Rope(D, rot, qb.ROPE_PAIRS if pairs else qb.ROPE_HALF, tab, 1.25)
    for inverse in (False, True):
        for x, y in zip((q, k), qb.rope(cfg, pos, q, k, inverse=inverse)):
            ref, bound = ref_rope(x, pos, table_turns(tab), rot, pairs, inverse, 1.25)
            if dtype == torch.bfloat16:
                bound = bound + 2.0 ** -8 * ref.abs()
            within(y, ref, bound, f"inverse={inverse}")


@pytest.mark.parametrize("off", [0, 1])
def test_rope_strided_views_in_place_and_mixed_types(off):
    # q and k are views of one fused tensor; `off` = 1 makes every row misaligned for wide loads
    qb = _qb()
    g = _gen(3)
    T, H, Hk, D = 19, 6, 2, 64
    raw = torch.randn(T, (H + 2 * Hk) * D + off, generator=g, device=DEV)
    view = lambda r, h0, h: r[:, off:].view(T, H + 2 * Hk, D)[:, h0:h0 + h] if off == 0 else torch.as_strided(  # noqa: E731
        r, (T, h, D), (r.stride(0), D, 1), off + h0 * D)
    pos = torch.arange(T, dtype=torch.int32, device=DEV) - 4            # negative positions turn backwards
    tab = qb.rope_table(D)
    cfg = qb.Rope(D, D, qb.ROPE_HALF, tab)
    refs = [ref_rope(view(raw, h0, h), pos, table_turns(tab), D, False) for h0, h in ((0, H), (H, Hk))]
    # fp32 in, bf16 out
    oq = torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV)
    qb.rope(cfg, pos, view(raw, 0, H), out_q=oq)
    within(oq, refs[0][0], refs[0][1] + 2.0 ** -8 * refs[0][0].abs())
    # in place; what lies beside the views is untouched
    keep = raw.clone()
    q, k = view(raw, 0, H), view(raw, H, Hk)
    qb.rope(cfg, pos, q, k, out_q=q, out_k=k)
    within(q, *refs[0])
    within(k, *refs[1])
    rest = view(raw, H + Hk, Hk)
    assert torch.equal(rest, view(keep, H + Hk, Hk))
    if off:
        assert torch.equal(raw[:, 0], keep[:, 0])
    # bf16 in, fp32 out
    qh = view(keep, 0, H).to(torch.bfloat16)
    of = torch.empty(T, H, D, device=DEV)
    qb.rope(cfg, pos, qh, out_q=of)
    ref, bound = ref_rope(qh, pos, table_turns(tab), D, False)
    within(of, ref, bound)


def test_rope_gradient_is_the_formulas_and_the_differences():
    # loss = sum(dy * rope(x)): its gradient is the inverse rotation of dy, and differences of the loss agree.  The rotation
    # is linear, so a central difference has no truncation error; in fp32 with step 1 its rounding error is below
    # 2 * n * 2^-24 * sum |dy y| / n terms -> 2^-20 * sum |dy||y| is a safe bound.
    qb = _qb()
    g = _gen(5)
    T, H, D, rot = 6, 3, 64, 48
    x = torch.randn(T, H, D, generator=g, device=DEV)
    dy = torch.randn(T, H, D, generator=g, device=DEV)
    pos = torch.tensor([0, 1, 17, 4095, 100001, 3], dtype=torch.int32, device=DEV)
    for layout in (qb.ROPE_HALF, qb.ROPE_PAIRS):
        cfg = qb.Rope(D, rot, layout, qb.rope_table(rot), 0.75)
        dx = qb.rope(cfg, pos, dy, inverse=True)[0]
        ref, bound = ref_rope(dy, pos, table_turns(cfg.table), rot, layout == qb.ROPE_PAIRS, True, 0.75)
        within(dx, ref, bound)
        loss = lambda z: float((qb.rope(cfg, pos, z)[0].double() * dy.double()).sum())  # noqa: E731
        size = float((dy.double().abs() * x.double().abs()).sum())
        for t, h, d in ((0, 0, 0), (1, 2, 47), (4, 1, 5), (5, 0, 63), (3, 1, 24)):
            up, dn = x.clone(), x.clone()
            up[t, h, d] += 1.0
            dn[t, h, d] -= 1.0
            assert abs((loss(up) - loss(dn)) / 2 - float(dx[t, h, d])) <= 2.0 ** -20 * size


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("order", ["nhd", "hnd"])
@pytest.mark.parametrize("T,H,Hk,D,rot,page", [(1, 8, 2, 128, 128, 16), (23, 4, 4, 64, 32, 16), (9, 3, 1, 40, 20, 5)])
def test_rope_append_writes_its_slots_and_nothing_else(dtype, order, T, H, Hk, D, rot, page):
    qb = _qb()
    g = _gen(T)
    q, k, v = (torch.randn(T, n, D, generator=g, device=DEV).to(dtype) for n in (H, Hk, Hk))
    pos = torch.randint(0, 5000, (T,), generator=g, device=DEV).to(torch.int32)
    ck, cv, _, _, _ = make_cache(g, [3 * page], page, Hk, D, order, fill=7.0, spare=4)
    kk, kv = ck.clone(), cv.clone()
    n_slots = ck.shape[0] * page
    slots = torch.randperm(n_slots, generator=g, device=DEV)[:T].to(torch.int32)
    if T > 2:
        slots[1], slots[2] = -1, n_slots                      # padding, and one past the cache: nothing is written
    tab = qb.rope_table(rot)
    oq = qb.rope_append(qb.Rope(D, rot, qb.ROPE_HALF, tab), pos, slots, q, k, v, qb.KVCache(ck, cv))
    rq, bq = ref_rope(q, pos, table_turns(tab), rot, False)
    rk, bk = ref_rope(k, pos, table_turns(tab), rot, False)
    within(oq, rq, bq + 2.0 ** -8 * rq.abs())
    ok = (slots >= 0) & (slots < n_slots)
    s = slots[ok].long()
    within(ck[s // page, s % page], rk[ok], (bk + 2.0 ** -8 * rk.abs())[ok])
    assert torch.equal(cv[s // page, s % page], v[ok].to(torch.bfloat16))
    kk[s // page, s % page] = ck[s // page, s % page]
    kv[s // page, s % page] = cv[s // page, s % page]
    assert torch.equal(ck, kk) and torch.equal(cv, kv)


# --------------------------------------------------------------------------------------------------------------- plan
def _ref_plan(ctx, new, gone, table, stack, n_free, page, T):
    """The header's definition, request by request, on Python lists."""
    B, width, cap = len(ctx), len(table[0]), len(stack)
    table, stack = [list(r) for r in table], list(stack)
    pages = lambda n: -(-n // page)  # noqa: E731
    free = n_free
    for b in range(B):
        if gone[b]:
            for j in range(pages(min(max(ctx[b], 0), width * page))):
                stack[free] = table[b][j]
                free += 1
    avail, taken, rows, cut = free, 0, 0, False
    cu, kv, pos, slots, adm = [0], [], [], [], []
    for b in range(B):
        c = min(max(ctx[b], 0), width * page)
        valid = not gone[b] and ctx[b] >= 0 and new[b] >= 0 and ctx[b] + new[b] <= width * page
        need, add = (pages(c + new[b]) - pages(c), new[b]) if valid else (0, 0)
        if valid and (taken + need > avail or rows + add > T):
            cut = True
        ok = valid and not cut
        if ok:
            for i in range(need):
                table[b][pages(c) + i] = stack[avail - 1 - taken - i]
            taken += need
            rows += add
            for p in range(c, c + add):
                pos.append(p)
                slots.append(table[b][p // page] * page + p % page)
        adm.append(int(ok))
        cu.append(rows)
        kv.append(0 if gone[b] else c + (add if ok else 0))
    pos += [0] * (T - rows)
    slots += [-1] * (T - rows)
    return dict(table=table, stack=stack, cu_new=cu, kv_len=kv, positions=pos, slots=slots, admitted=adm, free_count=[avail - taken])


def _run_plan(ctx, new, gone, page, T, width, n_free_extra, seed=0, with_release=True):
    qb = _qb()
    r = torch.Generator().manual_seed(seed)
    held = [-(-min(max(c, 0), width * page) // page) for c in ctx]
    total = sum(held) + max(n_free_extra, 0)
    perm = torch.randperm(max(total, 1), generator=r).tolist()
    table, at = [], 0
    for h in held:
        table.append(perm[at:at + h] + [-7] * (width - h))
        at += h
    n_free = total - sum(held)
    cap = max(total, 1)
    stack = perm[at:at + n_free] + [-9] * (cap - n_free)
    ref = _ref_plan(ctx, new, gone, table, stack, n_free, page, T)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    dt, ds, cnt = i32(table), i32(stack), i32([n_free])
    for again in range(2):                                            # a second call on the same inputs changes nothing
        p = qb.kv_plan(i32(ctx), i32(new), dt, ds, cnt, page, T, release=i32([int(x) for x in gone]) if with_release else None)
        got = dict(table=dt, stack=ds, cu_new=p.cu_new, kv_len=p.kv_len, positions=p.positions, slots=p.slots,
                   admitted=p.admitted, free_count=p.free_count)
        for name, want in ref.items():
            assert got[name].tolist() == want, (name, again)
    return ref


@pytest.mark.parametrize("page", [1, 5, 16, 64])
def test_plan_small_cases(page):
    _run_plan([0], [1], [0], page, 1, 4, 4, with_release=False)
    _run_plan([0], [0], [0], page, 1, 1, 0)
    _run_plan([page], [1], [0], page, 3, 4, 1)                         # a full page: the token opens a new one
    _run_plan([page - 1], [1], [0], page, 3, 4, 0)                     # the last entry of a page needs none
    ref = _run_plan([page, 3, 2 * page], [1, 1, 2 * page + 1], [0, 1, 0], page, 4 * page + 4, 8, 2)
    assert ref["admitted"][1] == 0 and ref["kv_len"][1] == 0


def test_plan_admission_is_first_come_first_served():
    # pages run out at the third request; the fourth, which needs none, waits as well
    ref = _run_plan([16, 16, 16, 3], [1, 1, 40, 1], [0, 0, 0, 0], 16, 64, 8, 3)
    assert ref["admitted"] == [1, 1, 0, 0]
    # rows run out
    ref = _run_plan([0, 0, 0], [5, 5, 1], [0, 0, 0], 16, 9, 8, 8)
    assert ref["admitted"] == [1, 0, 0]
    # invalid ones (negative lengths, wider than the table) do not hold up the others
    ref = _run_plan([-3, 4, 0, 5], [1, -1, 200, 2], [0, 0, 0, 0], 16, 9, 4, 8)
    assert ref["admitted"] == [0, 0, 0, 1]
    # pages given back in this very call are handed out in it
    ref = _run_plan([40, 0], [0, 48], [1, 0], 16, 48, 4, 0)
    assert ref["admitted"] == [0, 1] and ref["free_count"] == [0]


@pytest.mark.parametrize("seed", range(6))
def test_plan_random_steps(seed):
    r = torch.Generator().manual_seed(100 + seed)
    ri = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=r))  # noqa: E731
    B = [1, 31, 255, 256, 257, 1111][seed]
    page = [16, 1, 7, 32, 16, 16][seed]
    ctx = [ri(0, 90) for _ in range(B)]
    new = [ri(0, 3) if ri(0, 9) else ri(0, 200) for _ in range(B)]
    gone = [ri(0, 9) == 0 for _ in range(B)]
    width = -(-300 // page)
    want = sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(ctx, new))
    _run_plan(ctx, new, gone, page, sum(new) + 3, width, want if seed % 2 else want // 2, seed)


def test_plan_most_requests():
    r = torch.Generator().manual_seed(7)
    B = 8192
    ctx = torch.randint(0, 40, (B,), generator=r).tolist()
    new = torch.randint(0, 3, (B,), generator=r).tolist()
    ref = _run_plan(ctx, new, [b % 17 == 0 for b in range(B)], 16, sum(new), 4, 6000)
    assert ref["admitted"][-1] == 1


# ---------------------------------------------------------------------------------------------------------- attention
def _attend(new, kv, H, Hkv, D, page=16, order="nhd", causal=True, window=0, seed=1, scale=None, qstd=1.5, std=1.0, edit=None,
            q_view=False, fill=float("nan")):
    qb = _qb()
    g = _gen(seed)
    ck, cv, table, ks, vs = make_cache(g, kv, page, Hkv, D, order, std=std, fill=fill)
    T = sum(new)
    q = (torch.randn(max(T, 1), H, D, generator=g, device=DEV) * qstd).to(torch.bfloat16)
    if q_view:
        wide = torch.full((max(T, 1), H + 2, D + 8), 3.0, dtype=torch.bfloat16, device=DEV)
        wide[:, 1:1 + H, :D] = q
        q = wide[:, 1:1 + H, :D]
    if edit:
        edit(ks, vs, q, lambda b, j: (ck[int(table[b, j // page]), j % page], cv[int(table[b, j // page]), j % page]))
    scale = D ** -0.5 if scale is None else scale
    out = torch.full((max(T, 1) + 1, H, D), 5.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((max(T, 1), H), 5.0, device=DEV)
    cache = qb.KVCache(ck, cv)
    ws = qb.alloc_attention_workspace(cache, q)
    ws.fill_(0xA5)
    qb.paged_attention(q, cache, table, offsets(new), torch.tensor(kv, dtype=torch.int32, device=DEV), scale=scale,
                       causal=causal, window=window, out=out[:-1], lse=lse, ws=ws)
    assert qb.device_status(ws) == qb.OK
    assert bool((out[-1] == 5.0).all())
    ref, bound, rl, lb = ref_attention(q, ks, vs, new, kv, scale, causal, window)
    within(out[:T], ref[:T], bound[:T], "out")
    within(lse[:T], rl[:T], lb[:T], "lse")
    return out[:T], lse[:T]


HEADS = [(1, 1), (4, 1), (8, 8), (10, 2), (12, 4), (16, 1), (7, 1)]


@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("D", [64, 128])
def test_attention_single_tokens(H, Hkv, D):
    kv = [1, 2, 15, 16, 17, 31, 33, 127, 128, 129, 300, 1000]
    _attend([1] * len(kv), kv, H, Hkv, D)


@pytest.mark.parametrize("page", [1, 3, 8, 16, 32, 48, 64, 128, 256])
def test_attention_page_sizes(page):
    _attend([1, 5, 40, 1], [700, 131, 261, 5], 8, 2, 128, page=page)
    _attend([130], [260], 4, 4, 64, page=page)


@pytest.mark.parametrize("D", [8, 40, 64, 80, 96, 128, 192, 256])
def test_attention_head_sizes(D):
    _attend([1, 3, 20, 70], [50, 200, 20, 333], 4, 2, D)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,kv,H,Hkv", [
    ([1], [2000], 8, 1), ([1], [1], 4, 4), ([1], [513], 32, 8), ([4], [900], 32, 4), ([1], [700], 16, 16), ([1], [333], 34, 34),
    ([1], [129], 80, 80), ([1] * 6, [1, 0, 17, 400, 2, 96], 16, 4), ([0, 3, 0, 2, 1], [5, 3, 0, 700, 257], 15, 3),
    ([17, 1, 0, 14], [17, 300, 9, 5], 3, 3), ([1] * 9, [40 * i + 1 for i in range(9)], 21, 7), ([32], [33], 2, 2),
])
def test_attention_calls_of_few_rows(new, kv, H, Hkv, D):
    # every number of CTAs per key head, more of them than key tiles, row tiles that few requests have
    _attend(new, kv, H, Hkv, D)
    _attend(new, kv, H, Hkv, D, page=8, order="hnd", causal=False, seed=2)
    _attend(new, kv, H, Hkv, D, page=64, window=100, q_view=True, seed=3)


@pytest.mark.parametrize("new,kv", [([1], [5000]), ([2, 0, 1, 1], [900, 5, 1, 0]), ([1] * 5, [3000, 3, 17, 64, 2000])])
def test_attention_does_not_depend_on_the_tables_width(new, kv):
    # columns behind a request's pages are never read; a wide table's call may be worked on in another way
    qb = _qb()
    g = _gen(21)
    ck, cv, table, ks, vs = make_cache(g, kv, 16, 4, 128)
    q = torch.randn(sum(new), 16, 128, generator=g, device=DEV).to(torch.bfloat16)
    ref, bound, rl, lb = ref_attention(q, ks, vs, new, kv, 128 ** -0.5)
    for width in (table.shape[1], 1024, 9000, 100000):
        wide = torch.full((len(kv), width), -1, dtype=torch.int32, device=DEV)
        wide[:, :table.shape[1]] = table
        out, lse = qb.paged_attention(q, qb.KVCache(ck, cv), wide, offsets(new), torch.tensor(kv, dtype=torch.int32, device=DEV),
                                      need_lse=True)
        within(out, ref, bound, "out")
        within(lse, rl, lb, "lse")


@pytest.mark.parametrize("H,Hkv", HEADS)
def test_attention_chunks(H, Hkv):
    _attend([1, 37, 128, 1, 200], [600, 37, 129, 1, 777], H, Hkv, 128)
    _attend([65, 300], [65, 301], H, Hkv, 64)


@pytest.mark.parametrize("H,Hkv,D,new,kv", [
    (8, 8, 128, [900, 1, 333], [2900, 700, 333]),           # shares of many tiles that cross items and requests
    (16, 16, 64, [700, 650], [3000, 650]),
    (32, 4, 128, [500], [5000]),                             # shared keys
    (64, 64, 64, [2600], [2600]),                            # more than four items per SM: whole items
    (40, 40, 128, [1600, 1, 1700], [1700, 9, 1700]),
])
def test_attention_long_chunks(H, Hkv, D, new, kv):
    _attend(new, kv, H, Hkv, D)
    if H < 40:
        _attend(new, kv, H, Hkv, D, window=300, seed=2)
        _attend(new, kv, H, Hkv, D, page=128, causal=False, seed=3)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,kv,H,Hkv", [
    ([40], [20001], 1, 1),            # one row tile cut into as many parts as there are SMs
    ([200], [9000], 1, 1),            # two row tiles
    ([34, 1, 33], [129, 40, 3000], 2, 2), ([127], [128], 1, 1), ([128, 129], [256, 385], 1, 1),   # one key tile to each, or few
    ([11, 5, 40], [700, 2100, 900], 12, 3), ([300, 2], [4000, 3], 6, 2),
])
def test_attention_items_cut_many_times(new, kv, H, Hkv, D):
    _attend(new, kv, H, Hkv, D)
    _attend(new, kv, H, Hkv, D, page=32, causal=False, seed=2)
    _attend(new, kv, H, Hkv, D, page=128, window=500, q_view=True, seed=3)


@pytest.mark.parametrize("order", ["nhd", "hnd"])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 20), (True, 130), (False, 50), (True, 4000)])
def test_attention_masks_and_orders(order, causal, window):
    _attend([1, 30, 150, 2], [513, 333, 150, 2], 8, 2, 128, order=order, causal=causal, window=window, q_view=True)
    _attend([1] * 5, [513, 20, 21, 150, 2], 8, 8, 64, order=order, causal=causal, window=window)


def test_attention_rows_that_see_nothing():
    # more new rows than keys: the first rows lie in front of the sequence; requests without keys or without rows
    for H, Hkv in ((4, 1), (32, 8)):
        out, lse = _attend([3, 0, 5, 1, 90], [0, 40, 2, 7, 60], H, Hkv, 128)
        assert bool((out[:3] == 0).all()) and bool(torch.isneginf(lse[:3]).all())
        assert bool((out[3:6] == 0).all()) and bool(torch.isneginf(lse[3:6]).all())
        _attend([300], [10], H, Hkv, 64)
        _attend([1, 1], [0, 0], H, Hkv, 64)


def test_attention_large_scores_and_sinks():
    # scores of magnitude 100 and more: the running maximum moves by far more than the exponent range of a weight
    _attend([1, 9, 200], [400, 300, 900], 8, 2, 128, qstd=12.0, std=2.0)
    _attend([1, 9, 200], [400, 300, 900], 8, 2, 128, scale=-0.2)
    _attend([1, 9, 200], [400, 300, 900], 8, 2, 128, scale=0.0)

    def rising(ks, vs, q, at):               # keys that grow along the sequence: every tile has a new maximum
        for b in range(len(ks)):
            n = ks[b].shape[0]
            for j in range(n):
                ks[b][j] = (q[b if b < 2 else 10, 0].float() * (0.02 * j)).to(torch.bfloat16)
                at(b, j)[0][:] = ks[b][j]
    _attend([1, 9, 200], [400, 300, 500], 2, 1, 128, edit=rising)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new,kv", [([4], [60]), ([40], [200]), ([150], [400]), ([1], [70])])
def test_attention_masked_keys_hold_anything(bad, new, kv):
    # the newest key and value are not finite: rows that do not see them are exact, those that do follow the definition
    def plant(ks, vs, q, at):
        j = kv[0] - 1
        for t in (ks[0], at(0, j)[0].unsqueeze(0)):
            t[-1, 0, 3] = bad
        for t in (vs[0], at(0, j)[1].unsqueeze(0)):
            t[-1, 1, 5] = bad
    # every row but the last is finite
    qb = _qb()
    for H, Hkv in ((2, 2), (8, 2)):
        g = _gen(9)
        ck, cv, table, ks, vs = make_cache(g, kv, 16, Hkv, 128)
        at = lambda b, j: (ck[int(table[b, j // 16]), j % 16], cv[int(table[b, j // 16]), j % 16])  # noqa: E731
        q = torch.randn(new[0], H, 128, generator=g, device=DEV).to(torch.bfloat16)
        plant(ks, vs, q, at)
        out, lse = qb.paged_attention(q, qb.KVCache(ck, cv), table, offsets(new), torch.tensor(kv, dtype=torch.int32, device=DEV),
                                      need_lse=True)
        ref, bound, rl, lb = ref_attention(q[:-1], [k[:-1] for k in ks], [v[:-1] for v in vs], [new[0] - 1], [kv[0] - 1], 128 ** -0.5)
        within(out[:-1], ref, bound, "rows that do not see it")
        within(lse[:-1], rl, lb, "lse of rows that do not see it")
        G = H // Hkv
        if bad != bad:
            assert bool(out[-1, :G].isnan().all()) and bool(lse[-1, :G].isnan().all())     # NaN in a key it sees
            assert bool(out[-1, G:2 * G, 5].isnan().all())                                # NaN in a value it sees
        else:
            assert not bool(torch.isfinite(out[-1, G:2 * G, 5]).any())                    # an infinite value it sees
        keep = torch.ones(128, dtype=torch.bool, device=DEV)
        keep[5] = False
        assert bool(torch.isfinite(out[-1, G:2 * G][:, keep]).all())


@pytest.mark.parametrize("new", [1, 5, 60, 300])
def test_attention_seen_values_that_are_not_finite(new):
    # far from every mask: an infinite value reaches its column of every row, a NaN key every column
    qb = _qb()
    g = _gen(12)
    kv, H, Hkv, D = 900, 4, 2, 128
    ck, cv, table, ks, vs = make_cache(g, [kv], 16, Hkv, D, fill=0.0)
    at = lambda c, j: c[int(table[0, j // 16]), j % 16]  # noqa: E731
    at(cv, 200)[0, 7] = float("inf")
    at(ck, 333)[1, 64] = float("nan")
    q = torch.randn(new, H, D, generator=g, device=DEV).to(torch.bfloat16)
    out, lse = qb.paged_attention(q, qb.KVCache(ck, cv), table, offsets([new]), torch.tensor([kv], dtype=torch.int32, device=DEV),
                                  need_lse=True)
    assert not bool(torch.isfinite(out[:, :2, 7]).any())
    keep = torch.ones(D, dtype=torch.bool, device=DEV)
    keep[7] = False
    assert bool(torch.isfinite(out[:, :2][..., keep]).all()) and bool(torch.isfinite(lse[:, :2]).all())
    assert bool(out[:, 2:].isnan().all()) and bool(lse[:, 2:].isnan().all())


@pytest.mark.parametrize("new,kv", [([1, 1], [3000, 700]), ([6], [1500]), ([260, 40], [900, 640])])
@pytest.mark.parametrize("jump", [30.0, 300.0])
def test_attention_one_key_far_above_the_others(new, kv, jump):
    # one late key outgrows the maximum of the first tile by 2^43 or 2^433: weights of fp32's range and beyond it
    def plant(ks, vs, q, at):
        t = 0
        for b in range(len(new)):
            for j in (kv[b] // 2, kv[b] - new[b] - 1):
                u = q[t + new[b] // 2, 0].float()
                ks[b][j, 0] = (u * (jump * 128 ** 0.5 / float(u @ u))).to(torch.bfloat16)
                at(b, j)[0][0] = ks[b][j, 0]
            t += new[b]
    _attend(new, kv, 4, 1, 128, edit=plant, qstd=1.0, std=0.5)
    _attend(new, kv, 2, 1, 64, edit=plant, qstd=1.0, std=0.5)


@pytest.mark.parametrize("new,kv,D,window", [([1, 4, 40], [77, 130, 300], 128, 0), ([3, 20], [0, 64], 64, 9), ([2], [40], 24, 0)])
def test_attention_general_path(monkeypatch, new, kv, D, window):
    monkeypatch.setenv("QBLORA_FORCE_GENERAL", "1")
    _attend(new, kv, 6, 2, D, window=window)


def test_attention_on_two_streams_at_once():
    qb = _qb()
    g = _gen(21)
    jobs = []
    for new, kv in (([1] * 20, [1700] * 20), ([500], [2300])):
        ck, cv, table, _, _ = make_cache(g, kv, 32, 4, 128, fill=0.0)
        q = torch.randn(sum(new), 16, 128, generator=g, device=DEV).to(torch.bfloat16)
        cache = qb.KVCache(ck, cv)
        args = (q, cache, table, offsets(new), torch.tensor(kv, dtype=torch.int32, device=DEV))
        jobs.append((args, qb.alloc_attention_workspace(cache, q), torch.cuda.Stream(), qb.paged_attention(*args)[0]))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        for i, (args, ws, st, _) in enumerate(jobs):
            with torch.cuda.stream(st):
                outs[i].append(qb.paged_attention(*args, ws=ws)[0])
    torch.cuda.synchronize()
    for i, (_, ws, _, ref) in enumerate(jobs):
        assert all(torch.equal(o, ref) for o in outs[i])
        assert qb.device_status(ws) == qb.OK


def test_attention_on_another_stream_and_in_a_graph():
    # lengths and tables change between replays of one captured call
    qb = _qb()
    H, Hkv, D, page = 8, 2, 128, 16
    steps = [([1, 1, 1], [40, 900, 1]), ([70, 1, 0], [300, 33, 5]), ([1, 0, 70], [1, 0, 70])]
    T, width = 72, 64
    q = torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV)
    cache = qb.KVCache.empty(100, page, Hkv, D)
    table = torch.zeros(3, width, dtype=torch.int32, device=DEV)
    cu, kvl = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(T, H, device=DEV)
    ws = qb.alloc_attention_workspace(cache, q)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        qb.paged_attention(q, cache, table, cu, kvl, out=out, lse=lse, ws=ws)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            qb.paged_attention(q, cache, table, cu, kvl, out=out, lse=lse, ws=ws)
    for rep, (new, kv) in enumerate(steps * 2):
        g = _gen(rep)
        ck, cv, tb, ks, vs = make_cache(g, kv, page, Hkv, D, fill=0.0)
        with torch.cuda.stream(st):
            st.wait_stream(torch.cuda.default_stream())
            cache.k[:ck.shape[0]].copy_(ck)
            cache.v[:cv.shape[0]].copy_(cv)
            table[:, :tb.shape[1]].copy_(tb)
            cu.copy_(offsets(new))
            kvl.copy_(torch.tensor(kv, dtype=torch.int32))
            q.copy_(torch.randn(T, H, D, generator=g, device=DEV))
            graph.replay()
        st.synchronize()
        n = sum(new)
        ref, bound, rl, lb = ref_attention(q[:n], ks, vs, new, kv, D ** -0.5)
        within(out[:n], ref, bound, f"replay {rep}")
        within(lse[:n], rl, lb, f"replay {rep}")


def test_attention_repeats_bit_for_bit():
    a = _attend([1, 60, 300, 1], [5000, 700, 999, 2], 8, 2, 128)
    b = _attend([1, 60, 300, 1], [5000, 700, 999, 2], 8, 2, 128)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attention_page_number_out_of_range_is_reported():
    qb = _qb()
    g = _gen(2)
    for new in ([1], [200]):
        ck, cv, table, _, _ = make_cache(g, [400], 16, 2, 128, fill=0.0)
        table[0, 7] = 1 << 30
        q = torch.randn(new[0], 8, 128, generator=g, device=DEV).to(torch.bfloat16)
        cache = qb.KVCache(ck, cv)
        ws = qb.alloc_attention_workspace(cache, q)
        kv = torch.tensor([400], dtype=torch.int32, device=DEV)
        qb.paged_attention(q, cache, table, offsets(new), kv, ws=ws)
        assert qb.device_status(ws) == qb.ERR_INVALID_ARG
        table[0, 7] = -1
        qb.paged_attention(q, cache, table, offsets(new), kv, ws=ws)
        assert qb.device_status(ws) == qb.ERR_INVALID_ARG


@pytest.mark.parametrize("new", [[1], [0, 0], [1, 40]])
def test_attention_status_is_cleared_by_every_replay(new):
    qb = _qb()
    g = _gen(31)
    kv = [400] * len(new)
    ck, cv, table, ks, vs = make_cache(g, kv, 16, 2, 128, fill=0.0)
    q = torch.randn(max(sum(new), 1), 8, 128, generator=g, device=DEV).to(torch.bfloat16)
    cache = qb.KVCache(ck, cv)
    ws = qb.alloc_attention_workspace(cache, q)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    lens, cu = torch.tensor(kv, dtype=torch.int32, device=DEV), offsets(new)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        qb.paged_attention(q, cache, table, cu, lens, out=out, lse=lse, ws=ws)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            qb.paged_attention(q, cache, table, cu, lens, out=out, lse=lse, ws=ws)
        good = table[-1, 7].clone()
        for page, want in ((1 << 30, qb.ERR_INVALID_ARG), (good, qb.OK), (-1, qb.ERR_INVALID_ARG), (good, qb.OK)):
            table[-1, 7] = page
            out.fill_(5.0)
            ws[:4].fill_(0xFF)
            graph.replay()
            st.synchronize()
            assert qb.device_status(ws) == (want if sum(new) else qb.OK)
        if sum(new):
            ref, bound, rl, lb = ref_attention(q, ks, vs, new, kv, 128 ** -0.5)
            within(out, ref, bound, "out")
            within(lse, rl, lb, "lse")
        else:
            assert bool((out == 5.0).all())


@pytest.mark.parametrize("new", [1, 130])
def test_attention_offsets_past_32_bits(new):
    # a cache of 2.2e9 elements each for k and v: the request's pages lie at its end
    qb = _qb()
    page, Hkv, D = 64, 8, 128
    n_pages = (1 << 31) // (page * Hkv * D) + 900
    cache = qb.KVCache.empty(n_pages, page, Hkv, D)
    g = _gen(4)
    kv = 300
    ids = n_pages - 1 - torch.arange(5, device=DEV) * 3
    j = torch.arange(kv, device=DEV)
    ks = torch.randn(kv, Hkv, D, generator=g, device=DEV).to(torch.bfloat16)
    vs = torch.randn(kv, Hkv, D, generator=g, device=DEV).to(torch.bfloat16)
    slots = (ids[j // page] * page + j % page).to(torch.int32)
    zero = torch.zeros(kv, dtype=torch.int32, device=DEV)
    qb.rope_append(qb.Rope(D, D, qb.ROPE_HALF, qb.rope_table(D)), zero, slots, ks, ks, vs, cache)   # position 0: copied
    assert torch.equal(cache.k[ids[j // page], j % page], ks)
    q = torch.randn(new, 8, D, generator=g, device=DEV).to(torch.bfloat16)
    out, lse = qb.paged_attention(q, cache, ids.to(torch.int32)[None], offsets([new]), torch.tensor([kv], dtype=torch.int32, device=DEV),
                                  need_lse=True)
    ref, bound, rl, lb = ref_attention(q, [ks], [vs], [new], [kv], D ** -0.5)
    within(out, ref, bound)
    within(lse, rl, lb)


def test_refusals_on_device_tensors():
    qb = _qb()
    cache = qb.KVCache.empty(4, 16, 2, 128)
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    q = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(qb.QbloraError):                                   # query heads no multiple of the key heads
        qb.paged_attention(torch.zeros(3, 7, 128, dtype=torch.bfloat16, device=DEV), cache, i(1, 4), i(2), i(1))
    with pytest.raises(qb.QbloraError):                                   # fp32 queries
        qb.paged_attention(q.float(), cache, i(1, 4), i(2), i(1))
    with pytest.raises(ValueError):                                       # offsets too short
        qb.paged_attention(q, cache, i(2, 4), i(2), i(2))
    with pytest.raises(qb.QbloraError) as e:                              # workspace too small
        qb.paged_attention(q, cache, i(1, 4), i(2), i(1), ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == qb.ERR_WORKSPACE
    with pytest.raises(qb.QbloraError):
        qb.paged_attention(q, cache, i(1, 4), i(2), i(1), window=-1)
    tab = qb.rope_table(128)
    with pytest.raises(qb.QbloraError):
        qb.rope(qb.Rope(128, 130, qb.ROPE_HALF, torch.zeros(65, dtype=torch.int64, device=DEV)), i(3), q)
    with pytest.raises(ValueError):
        qb.rope(qb.Rope(128, 128, qb.ROPE_HALF, tab), i(2), q)
    with pytest.raises(qb.QbloraError):                                   # q_out must be bf16
        kv = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device=DEV)
        qb.rope_append(qb.Rope(128, 128, qb.ROPE_HALF, tab), i(3), i(3), q, kv, kv, cache, out_q=q.float())
    with pytest.raises(qb.QbloraError):                                   # the count in and out are two words
        cnt = i(1)
        qb.kv_plan(i(1), i(1), i(1, 4), i(8), cnt, 16, 4, outs=(i(2), i(1), i(4), i(4), i(1), cnt))
    torch.cuda.synchronize()


def test_a_merged_layer_decodes_as_it_would_over_the_whole_sequence():
    # quantized linears -> plan -> rotary + append -> attention -> linear, in chunks and single tokens, against the same layer
    # in 64 bits over each whole sequence.  The linears' bf16 outputs and the cache are shared, so what differs is rounding:
    # the rotated q and k (2^-8 each, on scores of size s: 2 * 2^-8 * s), the weights and the result, as in tests/_serving.py.
    qb = _qb()
    g = _gen(31)
    Dm, H, Hkv, D, page = 512, 8, 2, 64, 16
    W = [torch.randn(n, Dm, generator=g, device=DEV) * 0.06 for n in (H * D, Hkv * D, Hkv * D)]
    lin = [qb.quantize_blockwise(w, 64, 1, qb.FMT_AFFINE_MINMAX) for w in W]
    rope = qb.Rope(D, D, qb.ROPE_HALF, qb.rope_table(D))
    lens, B = [70, 3, 33], 3
    X = [torch.randn(n, Dm, generator=g, device=DEV).to(torch.bfloat16) for n in lens]
    cache = qb.KVCache.empty(24, page, Hkv, D)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    table, stack, count = i32([[-1] * 8] * B), torch.randperm(24, generator=g, device=DEV).to(torch.int32), i32([24])
    done, outs, proj = [0] * B, [[] for _ in range(B)], [[] for _ in range(B)]
    for step in range(40):
        new = [min(n - d, 40 if step == 0 else 1) for n, d in zip(lens, done)]
        if not sum(new):
            break
        T = sum(new) + 2
        plan = qb.kv_plan(i32(done), i32(new), table, stack, count, page, T)
        count = plan.free_count
        rows = torch.cat([X[b][done[b]:done[b] + new[b]] for b in range(B)] + [torch.zeros(2, Dm, dtype=torch.bfloat16, device=DEV)])
        q, k, v = (qb.lowbit_gemm(w, rows).view(T, -1, D) for w in lin)
        rq = qb.rope_append(rope, plan.positions, plan.slots, q, k, v, cache)
        o, _ = qb.paged_attention(rq, cache, table, plan.cu_new, plan.kv_len)
        assert plan.admitted.tolist() == [1] * B
        t = 0
        for b in range(B):
            outs[b].append(o[t:t + new[b]])
            proj[b].append((q[t:t + new[b]], k[t:t + new[b]], v[t:t + new[b]]))
            t += new[b]
            done[b] += new[b]
    assert done == lens
    for b in range(B):
        q, k, v = (torch.cat([p[i] for p in proj[b]]) for i in range(3))
        pos = torch.arange(lens[b], device=DEV)
        rq, _ = ref_rope(q, pos, table_turns(rope.table), D, False)
        rk, _ = ref_rope(k, pos, table_turns(rope.table), D, False)
        ref, bound, _, _ = ref_attention(rq, [rk], [v], [lens[b]], [lens[b]], D ** -0.5)
        S = torch.einsum("nhd,jhd->hnj", rq.abs(), rk.repeat_interleave(H // Hkv, 1).abs()).amax(-1).T * D ** -0.5
        A = v.double().abs().amax()                                            # no weighted mean of |v| exceeds the largest |v|
        within(torch.cat(outs[b]), ref, bound + (2.0 ** -7 * S)[..., None] * 2 * A, f"request {b}")


@pytest.mark.parametrize("D,new,kv", [(64, [3, 1], [40, 7]), (128, [2], [33]), (64, [5], [900])])
def test_attention_more_key_heads_than_warps(D, new, kv):
    # eight warps per SM stream the cache; one, a few and many key heads more than that, and as many
    warps = 8 * torch.cuda.get_device_properties(0).multi_processor_count
    for Hkv in (warps, warps + 1, warps + 96):
        _attend(new, kv, Hkv, Hkv, D)


@pytest.mark.parametrize("general", [False, True])
@pytest.mark.parametrize("page,D", [(8, 64), (8, 128), (16, 64), (16, 128), (64, 128), (24, 128), (5, 40)])
@pytest.mark.parametrize("new,kv,window", [
    ([1], [700], 30), ([2, 1], [513, 90], 9), ([1] * 40, [37 * i + 1 for i in range(40)], 100), ([40, 3], [900, 333], 77),
    ([200, 1], [1500, 640], 1), ([150], [150], 20), ([300], [2000], 500),
])
def test_attention_pages_in_front_of_the_window_may_be_gone(monkeypatch, general, page, D, new, kv, window):
    # a server gives pages back that lie wholly in front of the window: their entries hold no page number any more
    qb = _qb()
    if general:
        monkeypatch.setenv("QBLORA_FORCE_GENERAL", "1")
    H, Hkv = 6, 2
    g = _gen(41)
    ck, cv, table, ks, vs = make_cache(g, kv, page, Hkv, D)
    q = torch.randn(sum(new), H, D, generator=g, device=DEV).to(torch.bfloat16)
    gone = 0
    for b, (n, L) in enumerate(zip(new, kv)):
        e = max(0, L - n - window + 1) // page
        table[b, :e] = -1 if b % 2 else 1 << 30
        gone += e
    assert gone or max(kv) == 150
    cache = qb.KVCache(ck, cv)
    ws = qb.alloc_attention_workspace(cache, q)
    out, lse = qb.paged_attention(q, cache, table, offsets(new), torch.tensor(kv, dtype=torch.int32, device=DEV), window=window,
                                  need_lse=True, ws=ws)
    assert qb.device_status(ws) == qb.OK
    ref, bound, rl, lb = ref_attention(q, ks, vs, new, kv, D ** -0.5, window=window)
    within(out, ref, bound, "out")
    within(lse, rl, lb, "lse")


def test_calls_on_a_stream_own_their_memory_there(monkeypatch):
    # what a call on another stream allocates (workspaces above all, which it drops when it returns) comes from that stream's
    # memory: taken from the current stream's, the next tensor made there could lie in it while the kernels still run
    qb = _qb()
    g = _gen(51)
    kv, D = [900, 40, 300], 128
    new = [1, 40, 3]
    ck, cv, table, ks, vs = make_cache(g, kv, 16, 2, D, fill=0.0)
    q = torch.randn(sum(new), 8, D, generator=g, device=DEV).to(torch.bfloat16)
    k = torch.randn(sum(new), 2, D, generator=g, device=DEV).to(torch.bfloat16)
    cache, cu, lens = qb.KVCache(ck, cv), offsets(new), torch.tensor(kv, dtype=torch.int32, device=DEV)
    rope = qb.Rope(D, D, qb.ROPE_HALF, qb.rope_table(D))
    pos, slots = torch.zeros(sum(new), dtype=torch.int32, device=DEV), torch.full((sum(new),), -1, dtype=torch.int32, device=DEV)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    ctx, one, tab, free, count = i32([3]), i32([1]), i32([[0, -1]]), i32([1, 2]), i32([2])
    x = torch.randn(3, 256, generator=g, device=DEV).to(torch.bfloat16)
    w = torch.randn(128, 256, generator=g, device=DEV)
    ad = qb.Adapter(64, 8, 4, 1.0, torch.randn(4, 4, generator=g, device=DEV).bfloat16(), torch.randn(4, 16, generator=g, device=DEV).bfloat16())
    qw = qb.quantize_blockwise(w, 64, 1, qb.FMT_AFFINE_MINMAX)
    q2, wb = qb.quantize_minmax_nbit(w, 2), w.bfloat16()
    dy = torch.randn(3, 128, generator=g, device=DEV).to(torch.bfloat16)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    made, real = [], torch.empty

    def empty(*a, **kw):
        made.append(torch.cuda.current_stream().cuda_stream)
        return real(*a, **kw)

    calls = [lambda s: qb.paged_attention(q, cache, table, cu, lens, need_lse=True, stream=s), lambda s: qb.rope(rope, pos, q, k, stream=s),
             lambda s: qb.rope_append(rope, pos, slots, q, k, k, cache, stream=s),
             lambda s: qb.kv_plan(ctx, one, tab, free, count, 16, 2, stream=s), lambda s: qb.linear_fwd(qw, ad, x, stream=s),
             lambda s: qb.linear_bwd(qw, ad, x, dy, stream=s), lambda s: qb.merge(qw, ad, stream=s), lambda s: qb.merge_dense(qw, ad, stream=s),
             lambda s: qb.lowbit_gemm(qw, x, stream=s), lambda s: qb.dense_gemm(wb, x, stream=s),
             lambda s: qb.quantize_blockwise(w, 64, 1, qb.FMT_AFFINE_MINMAX, stream=s), lambda s: qb.quantize_minmax_nbit(w, 2, stream=s),
             lambda s: qb.unpack_codes(qb.pack_codes(q2, 2, stream=s), stream=s)]
    monkeypatch.setattr(torch, "empty", empty)
    for i, call in enumerate(calls):
        made.clear()
        call(side)
        torch.cuda.synchronize()
        assert made and set(made) == {side.cuda_stream}, (i, made)
    monkeypatch.undo()

    # and the results are right while the current stream takes and overwrites memory of the workspace's size at once
    ref, bound, rl, lb = ref_attention(q, ks, vs, new, kv, D ** -0.5)
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(side):
            torch.cuda._sleep(2000000)
        out, lse = qb.paged_attention(q, cache, table, cu, lens, need_lse=True, stream=side)
        real(qb.attention_workspace_bytes(cache, 8, sum(new)), dtype=torch.uint8, device=DEV).fill_(0x7F)
        torch.cuda.synchronize()
        within(out, ref, bound, "out")
        within(lse, rl, lb, "lse")


def test_workspaces_that_are_smaller_than_they_look_are_refused():
    qb = _qb()
    cache = qb.KVCache.empty(4, 16, 2, 128)
    q = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device=DEV)
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    for ws in (torch.empty(1, dtype=torch.uint8, device=DEV).expand(1 << 30), torch.empty(1 << 20, dtype=torch.uint8, device=DEV)[::2],
               torch.empty(1 << 30, dtype=torch.uint8), torch.empty(1 << 20, device=DEV)):
        with pytest.raises(ValueError):
            qb.paged_attention(q, cache, i(1, 4), i(2), i(1), ws=ws)


@pytest.mark.parametrize("size", [2.0 ** 100, 2.0 ** -100])
@pytest.mark.parametrize("run", [16, 32, 128, 300])
@pytest.mark.parametrize("D,new,kv", [(128, [1], [4000]), (64, [1, 1, 1, 1], [2000, 900, 40, 600]), (128, [1] * 40, [900] * 40),
                                      (128, [20, 3], [900, 333]), (64, [150], [1500]), (128, [300, 40], [1000, 700]), (96, [5], [700])])
def test_attention_large_and_small_values_under_rising_scores(size, run, D, new, kv):
    # runs of keys with scores 26 above the ones in front of them (weights up to 2^37 of theirs), and values whose products with
    # such weights would leave the range of fp32: the result is a weighted mean of the values and stays within theirs
    def plant(ks, vs, q, at):
        g = _gen(7)
        u = torch.randn(D, generator=g, device=DEV)
        u *= (D / float(u @ u)) ** 0.5
        q.copy_((u + 0.05 * torch.randn(q.shape, generator=g, device=DEV)).to(torch.bfloat16))
        for b in range(len(ks)):
            for j in range(kv[b]):
                ks[b][j] = (u * (26.0 * (j // run % 2) / D ** 0.5)).to(torch.bfloat16)
                vs[b][j] *= size
                k, v = at(b, j)
                k.copy_(ks[b][j])
                v.copy_(vs[b][j])
    _attend(new, kv, 8, 2, D, edit=plant)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [3, 5, 7, 24])
def test_attention_does_not_depend_on_what_shared_memory_held(G, D):
    # G does not divide 128, so the last rows of a query tile are never filled; and a request's last tile holds rows of the next
    # request.  Neither may have a say in how the rows that are there are worked on: results are equal bit for bit.
    qb = _qb()
    g = _gen(61)
    new, kv = [300, 50], [900, 700]
    ck, cv, table, ks, vs = make_cache(g, kv, 16, 4, D)
    q = torch.randn(sum(new), 4 * G, D, generator=g, device=DEV).to(torch.bfloat16)
    args = (qb.KVCache(ck, cv), table, offsets(new), torch.tensor(kv, dtype=torch.int32, device=DEV))
    pk, pv, ptable, _, _ = make_cache(g, [512], 16, 64, D, fill=0.0)
    outs = []
    for held in (0.0, float("nan"), 3e38, 1.0):
        fill = torch.full((512, 64, D), held, dtype=torch.bfloat16, device=DEV)          # 128 items: most SMs' query tiles
        qb.paged_attention(fill, qb.KVCache(pk, pv), ptable, offsets([512]), torch.tensor([512], dtype=torch.int32, device=DEV))
        outs.append(qb.paged_attention(q, *args, need_lse=True))
        other = q.clone()
        other[300:] = held                                                              # the second request's queries
        outs.append([t[:300] for t in qb.paged_attention(other, *args, need_lse=True)])
    for out, lse in outs:
        assert torch.equal(out[:300], outs[0][0][:300]) and torch.equal(lse[:300], outs[0][1][:300])
    ref, bound, rl, lb = ref_attention(q, ks, vs, new, kv, D ** -0.5)
    within(outs[0][0], ref, bound, "out")
    within(outs[0][1], rl, lb, "lse")


@pytest.mark.parametrize("window", [(1 << 31) - 1, (1 << 31) - 3])
def test_attention_widest_windows(monkeypatch, window):
    # a window that never ends, also for rows in front of the sequence (fewer keys than new rows)
    for new, kv in (([6], [2]), ([1, 9], [40, 3]), ([300], [10]), ([70, 1], [5, 900])):
        for causal in (True, False):
            _attend(new, kv, 4, 2, 128, causal=causal, window=window)
            _attend(new, kv, 4, 2, 40, causal=causal, window=window)
    monkeypatch.setenv("QBLORA_FORCE_GENERAL", "1")
    _attend([6], [2], 4, 2, 64, causal=False, window=window)


@pytest.mark.parametrize("B", [257, 300, 385, 500, 1024, 1025, 1500])
@pytest.mark.parametrize("D,H,Hkv,window", [(64, 4, 2, 0), (128, 3, 1, 25)])
def test_attention_calls_of_many_requests(B, D, H, Hkv, window):
    # more requests than a CTA has threads (256 in the line form, 384 in the tcgen05 form), than the tcgen05 form lists (1024); with
    # and without prompts among them
    kv = [(37 * b) % 150 for b in range(B)]
    new = [min(b % 4, kv[b]) for b in range(B)]
    _attend(new, kv, H, Hkv, D, window=window, seed=B)
    for b, n in ((B // 2, 150), (B - 2, 400), (3, 40)):
        new[b], kv[b] = n, n + 70 * (b % 3)
    _attend(new, kv, H, Hkv, D, window=window, seed=B + 1)
    new = [max(1, b % 23) for b in range(B)] if B <= 500 else new                      # and many of either kind
    _attend(new, [n + 30 for n in new], H, Hkv, D, page=32, window=window, seed=B + 2)


def test_the_serving_example_runs():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    cmd = [sys.executable, os.path.join(root, "examples", "serve_layer.py"), "--hidden", "512", "--heads", "8", "--kv-heads", "2",
           "--dim", "64", "--prompts", "70,3,130", "--steps", "6"]
    done = subprocess.run(cmd, capture_output=True, text=True, timeout=240, cwd=root)
    assert done.returncode == 0, done.stderr[-2000:]
    assert "[75, 8, 135] cached tokens" in done.stdout
