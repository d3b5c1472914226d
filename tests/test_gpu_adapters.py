"""Many adapters over one weight on the GPU: plan, forward, backward against 64-bit forms, both paths, awkward batches."""
import random

import pytest
import torch

from tests import _adapters as ra
from tests._adapters import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_b200 import binding
    return binding


def _randn(seed, *shape, dtype=torch.bfloat16, gain=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * gain).to(dtype)


# ------------------------------------------------------------------------------------------------------------------ plan
PLANS = [([1], [0], 1, 1), ([5], [-1], 3, 9), ([0, 0], [0, 1], 2, 1), ([3, 0, 4, 1], [1, 0, 1, 7], 2, 8),
         ([1] * 33, [2] * 33, 3, 40), ([1] * 700, None, 100, 700), ([7, 300, 1, 1, 64] * 30, None, 9, 11200), ([1] * 8192, None, 4096, 8192),
         ([2] * 8192, [5] * 8192, 6, 16384), ([100000, 1, 50000], [1, 0, 1], 2, 150010)]


@pytest.mark.parametrize("lengths,ids,n,tokens", PLANS, ids=[str(i) for i in range(len(PLANS))])
def test_plan(qb, lengths, ids, n, tokens):
    r = random.Random(len(lengths) + n)
    ids = ids if ids is not None else [r.randrange(-1, n) for _ in lengths]
    cu, di, _ = ra.requests(lengths, ids)
    rows, start = (torch.full((k + 8,), 77, dtype=torch.int32, device=DEV) for k in (tokens, n + 1))
    p = qb.adapter_plan(cu, di, n, tokens, outs=(rows, start))
    want_rows, want_start = ra.ref_plan(cu.tolist(), ids, n, tokens)
    assert p.rows.tolist() == want_rows + [77] * 8 and p.start.tolist() == want_start + [77] * 8
    again = qb.adapter_plan(cu, di, n, tokens)
    assert torch.equal(again.rows, rows[:tokens]) and torch.equal(again.start, start[:n + 1])


def test_plan_offsets_out_of_range_stay_inside(qb):
    # offsets that fall, pass the buffer or are negative: nothing outside rows and start is written, start stays in range
    for cu in ([0, 50, 20, 900, 30], [-5, 3, 4, 4, 4], [0, 2 ** 31 - 1, 0, 2 ** 31 - 1, 7], [60, 61, 62, 63, 64]):
        rows, start = (torch.full((k + 8,), 77, dtype=torch.int32, device=DEV) for k in (64, 4))
        qb.adapter_plan(torch.tensor(cu, dtype=torch.int32, device=DEV), torch.tensor([0, 1, 2, 1], dtype=torch.int32, device=DEV), 3, 64,
                        outs=(rows, start))
        assert rows[64:].tolist() == [77] * 8 and start[4:].tolist() == [77] * 8
        assert all(0 <= v <= 64 for v in start[:4].tolist()) and all(v == 77 or -1 <= v < 64 for v in rows[:64].tolist())


# ---------------------------------------------------------------------------------------------------- forward and backward
#          d_in  d_out  l1  l2   r
SIZES = [(256, 512, 64, 8, 32), (512, 256, 4, 4, 64), (128, 128, 1, 1, 16), (1024, 1024, 64, 8, 256), (640, 1152, 2, 16, 48), (1024, 384, 8, 2, 8),
         (320, 272, 5, 2, 24), (96, 176, 3, 11, 40), (2048, 2048, 1, 1, 128), (4096, 512, 64, 64, 112),
         (60, 36, 4, 4, 7), (256, 260, 4, 4, 16), (130, 34, 2, 2, 3), (64, 64, 8, 8, 300)]       # the last four: general path
LENGTHS = {"one": ([1], [0], 1), "none": ([3, 2], [-1, -1], 2), "decode": ([1] * 40, None, 7), "empty": ([0, 1, 0, 5, 0], [1, 2, 0, 2, 3], 4),
           "tiles": ([16, 17, 15, 32, 33, 1, 64, 65], [0, 1, 2, 3, 4, 5, 6, 7], 9), "wide": ([127, 128, 129, 300, 2], [3, 0, 2, 1, 2], 4),
           "one adapter": ([200, 1, 77], [1, 1, 1], 2), "mixed": ([1] * 20 + [150] + [1] * 9, None, 5),
           "long": ([33, 1, 47, 48, 49, 9, 63, 64, 65, 300, 32], [0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 1], 11)}


CASES = [(size, lengths, dtype, general) for size in SIZES for lengths in LENGTHS for dtype in (torch.float32, torch.bfloat16)
         for general in (False, True) if not general or (lengths in ("tiles", "empty") and dtype is torch.float32)]
IDS = ["-".join(map(str, c[0])) + " " + c[1] + (" f32" if c[2] is torch.float32 else " bf16") + (" general" if c[3] else "") for c in CASES]


def _case(qb, size, lengths, seed, ranks=None, slack=3):
    lens, ids, n = LENGTHS[lengths]
    r = random.Random(seed)
    ids = ids if ids is not None else [r.randrange(-1, n) for _ in lens]
    bank = ra.make_bank(qb, n, *size, ranks=ranks, seed=seed)
    cu, di, T = ra.requests(lens, ids, sum(lens) + slack)
    return bank, cu.tolist(), ids, qb.adapter_plan(cu, di, n, T), T


def _paths(monkeypatch, general):
    if general:
        monkeypatch.setenv("QBLORA_FORCE_GENERAL", "1")


@pytest.mark.parametrize("size,lengths,dtype,general", CASES, ids=IDS)
def test_forward(qb, monkeypatch, size, lengths, dtype, general):
    _paths(monkeypatch, general)
    bank, cu, ids, plan, T = _case(qb, size, lengths, 11)
    X, Y0 = _randn(1, T, size[0]), _randn(2, T, size[1], dtype=dtype)
    Y = qb.adapters_fwd(bank, plan, X, Y0.clone())
    want, bound = ra.ref_fwd(bank, cu, ids, X, Y0)
    ra.check(Y, want, bound, 2, size[0] + size[4], ("Y", dtype), Y0)
    touched = torch.zeros(T, dtype=torch.bool, device=DEV)
    for b, a in enumerate(ids):
        touched[cu[b]:cu[b + 1]] = a >= 0
    assert torch.equal(Y[~touched], Y0[~touched])            # bit for bit


@pytest.mark.parametrize("size,lengths,dtype,general", CASES, ids=IDS)
def test_backward(qb, monkeypatch, size, lengths, dtype, general):
    _paths(monkeypatch, general)
    bank, cu, ids, plan, T = _case(qb, size, lengths, 12)
    X, dY, dX0 = _randn(3, T, size[0]), _randn(4, T, size[1]), _randn(5, T, size[0], dtype=dtype)
    nan = lambda t: torch.full(t.shape, float("nan"), device=DEV)  # noqa: E731
    dX, dA, dB = qb.adapters_bwd(bank, plan, X, dY, dX0.clone(), outs=(nan(bank.A), nan(bank.B)))
    want, bound = ra.ref_bwd(bank, cu, ids, X, dY, dX0)
    ra.check(dX, want[0], bound[0], 2, size[1] + size[4], ("dX", dtype), dX0)
    ra.check(dA, want[1], bound[1], 4, size[1] + size[0] // size[2] + T, ("dA", torch.float32))
    ra.check(dB, want[2], bound[2], 4, size[0] + size[1] // size[3] + T, ("dB", torch.float32))
    touched = torch.zeros(T, dtype=torch.bool, device=DEV)
    for b, a in enumerate(ids):
        touched[cu[b]:cu[b + 1]] = a >= 0
    assert torch.equal(dX[~touched], dX0[~touched])
    # parts alone are the same bits
    only = qb.adapters_bwd(bank, plan, None, dY, dX0.clone(), outs=(None, None))
    assert torch.equal(only[0], dX) and only[1] is None and only[2] is None
    assert torch.equal(qb.adapters_bwd(bank, plan, X, dY, None, need_db=False)[1], dA)
    assert torch.equal(qb.adapters_bwd(bank, plan, X, dY, None, need_da=False)[2], dB)


@pytest.mark.parametrize("general", [False, True], ids=["fast", "general"])
def test_uneven_ranks_and_what_lies_behind_them(qb, monkeypatch, general):
    # columns and rows from the rank (rounded up to 16) on are not read: they may hold anything
    _paths(monkeypatch, general)
    size = (512, 512, 4, 8, 64)
    ranks = [0, 1, 16, 17, 33, 48, 64, 200, -3]
    n = len(ranks)
    bank = ra.make_bank(qb, n, *size, ranks=[max(0, min(k, 64)) for k in ranks], seed=5)
    bank.ranks.copy_(torch.tensor(ranks, dtype=torch.int32))
    lens = [3, 20, 130, 1, 40, 17, 2, 9, 4]
    cu, di, T = ra.requests(lens, list(range(n)))
    plan = qb.adapter_plan(cu, di, n, T)
    X, dY, Y0, dX0 = _randn(1, T, 512), _randn(2, T, 512), _randn(3, T, 512, dtype=torch.float32), _randn(4, T, 512, dtype=torch.float32)
    want, bound = ra.ref_fwd(bank, cu.tolist(), list(range(n)), X, Y0)
    wantb, boundb = ra.ref_bwd(bank, cu.tolist(), list(range(n)), X, dY, dX0)
    for a, k in enumerate(ranks):
        k16 = (max(k, 0) + 15) // 16 * 16
        bank.A[a, :, k16:] = float("nan")
        bank.B[a, k16:] = float("inf")
        wantb[1][a, :, k16:] = 0
        wantb[2][a, k16:] = 0
    ra.check(qb.adapters_fwd(bank, plan, X, Y0.clone()), want, bound, 2, 576, ("Y", torch.float32), Y0)
    dX, dA, dB = qb.adapters_bwd(bank, plan, X, dY, dX0.clone())
    ra.check(dX, wantb[0], boundb[0], 2, 576, ("dX", torch.float32), dX0)
    ra.check(dA, wantb[1], boundb[1], 4, 1024 + T, ("dA", torch.float32))
    ra.check(dB, wantb[2], boundb[2], 4, 1024 + T, ("dB", torch.float32))


@pytest.mark.parametrize("general", [False, True], ids=["fast", "general"])
def test_strided_rows_and_what_lies_around_them(qb, monkeypatch, general):
    # q's and k's columns of one wide product, rows of a larger buffer
    _paths(monkeypatch, general)
    bank, cu, ids, plan, T = _case(qb, (256, 512, 4, 4, 32), "mixed", 3)
    X, big, grad = _randn(1, T, 256 * 3), _randn(2, T, 1536), _randn(3, T, 512 * 3, dtype=torch.float32)
    keep, keep_g = big.clone(), grad.clone()
    x, y = X[:, 256:512], big[:, 512:1024]
    want, bound = ra.ref_fwd(bank, cu, ids, x, y)
    qb.adapters_fwd(bank, plan, x, y)
    ra.check(y, want, bound, 2, 288, ("Y", torch.bfloat16))
    assert torch.equal(big[:, :512], keep[:, :512]) and torch.equal(big[:, 1024:], keep[:, 1024:])
    dY, dx = keep[:, 512:1024], grad[:, 512:768]
    want, bound = ra.ref_bwd(bank, cu, ids, x, dY, dx)
    _, dA, dB = qb.adapters_bwd(bank, plan, x, dY, dx)
    ra.check(dx, want[0], bound[0], 2, 544, ("dX", torch.float32), keep_g[:, 512:768])
    ra.check(dA, want[1], bound[1], 4, 600 + T, ("dA", torch.float32))
    ra.check(dB, want[2], bound[2], 4, 600 + T, ("dB", torch.float32))
    assert torch.equal(grad[:, :512], keep_g[:, :512]) and torch.equal(grad[:, 768:], keep_g[:, 768:])


def test_unaligned_tensors_take_the_general_path(qb):
    bank, cu, ids, plan, T = _case(qb, (256, 256, 4, 4, 32), "tiles", 4)
    X = _randn(1, T * 256 + 1)[1:].view(T, 256)
    Y = _randn(2, T * 257, dtype=torch.float32).view(T, 257)[:, 1:]
    want, bound = ra.ref_fwd(bank, cu, ids, X, Y)
    base = Y.clone()
    qb.adapters_fwd(bank, plan, X, Y)
    ra.check(Y, want, bound, 2, 288, ("Y", torch.float32), base)
    odd = qb.AdapterBank(256, 256, 4, 4, torch.empty(bank.A.numel() + 1, dtype=torch.bfloat16, device=DEV)[1:].view(bank.A.shape), bank.B,
                         bank.scaling)
    odd.A.copy_(bank.A)
    Y = base.clone()
    qb.adapters_fwd(odd, plan, X.clone(), Y)
    ra.check(Y, want, bound, 2, 288, ("Y", torch.float32), base)


@pytest.mark.parametrize("lengths", ["decode", "wide", "mixed"])
def test_values_that_are_not_finite_stay_in_their_rows(qb, lengths):
    bank, cu, ids, plan, T = _case(qb, (512, 512, 4, 4, 64), lengths, 6)
    X, Y0 = _randn(1, T, 512), _randn(2, T, 512, dtype=torch.float32)
    clean = qb.adapters_fwd(bank, plan, X, Y0.clone())
    bad = [b for b, a in enumerate(ids) if a >= 0][1]
    t = cu[bad + 1] - 1
    X[t, 100] = float("nan")
    got = qb.adapters_fwd(bank, plan, X, Y0.clone())
    other = torch.arange(T, device=DEV) != t
    assert torch.equal(got[other], clean[other]) and bool(got[t].isnan().all())
    # an adapter that holds NaN reaches its own rows alone
    X = _randn(1, T, 512)
    a = ids[bad]
    bank.B[a, 3, 7] = float("nan")
    got = qb.adapters_fwd(bank, plan, X, Y0.clone())
    mine = torch.zeros(T, dtype=torch.bool, device=DEV)
    for b, k in enumerate(ids):
        if k == a:
            mine[cu[b]:cu[b + 1]] = True
    assert torch.equal(got[~mine], clean[~mine]) and bool(got[mine][:, 28:32].isnan().all()) and torch.equal(got[mine][:, 32:], clean[mine][:, 32:])
    # and its gradients alone
    dY = _randn(3, T, 512)
    _, dA, dB = qb.adapters_bwd(bank, plan, X, dY)
    rest = torch.arange(bank.A.shape[0], device=DEV) != a
    assert bool(torch.isfinite(dA[rest]).all()) and bool(torch.isfinite(dB[rest]).all()) and bool(dA[a, :, 3].isnan().all())


def test_plan_entries_out_of_range_are_passed_over(qb):
    bank, cu, ids, plan, T = _case(qb, (256, 256, 4, 4, 32), "wide", 7)
    X, Y0 = _randn(1, T, 256), _randn(2, T, 256)
    want = qb.adapters_fwd(bank, plan, X, Y0.clone())
    rows = plan.rows.clone()
    rows[5], rows[200] = T + 9, -7
    got = qb.adapters_fwd(bank, qb.AdapterPlan(rows, plan.start), X, Y0.clone())
    lost = plan.rows[[5, 200]].long()
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[lost] = False
    assert torch.equal(got[keep], want[keep]) and torch.equal(got[lost], Y0[lost])
    # offsets past the buffer are clamped; an adapter between falling ones has no rows
    qb.adapters_fwd(bank, qb.AdapterPlan(plan.rows, plan.start + 100000), X, Y0.clone())
    start = plan.start.clone()
    start[1] = -4
    qb.adapters_fwd(bank, qb.AdapterPlan(plan.rows, start), X, Y0.clone())
    qb.adapters_bwd(bank, qb.AdapterPlan(rows, start.flip(0).contiguous()), X, _randn(3, T, 256), Y0.clone())
    torch.cuda.synchronize()


def test_gradients_against_differences(qb):
    # f(A, B, X) = sum of Y * W for the forward call in fp32; central differences of it along random directions, in 64 bits' formula
    bank, cu, ids, plan, T = _case(qb, (256, 512, 4, 8, 32), "mixed", 8)
    X, W = _randn(1, T, 256), _randn(2, T, 512)
    _, dA, dB = qb.adapters_bwd(bank, plan, X, W)
    dX = qb.adapters_bwd(bank, plan, X, W, torch.zeros(T, 256, device=DEV), outs=(None, None))[0]
    f = lambda A, B, x: float((ra.ref_fwd(qb.AdapterBank(256, 512, 4, 8, A, B, bank.scaling), cu, ids, x,  # noqa: E731
                                          torch.zeros(T, 512, device=DEV))[0] * W.double()).sum())
    for k, (t, grad) in enumerate(((bank.A, dA), (bank.B, dB), (X, dX))):
        v = _randn(20 + k, *t.shape, dtype=torch.float64)
        args = [bank.A.double(), bank.B.double(), X.double()]
        plus, minus = list(args), list(args)
        plus[k], minus[k] = args[k] + 1e-3 * v, args[k] - 1e-3 * v
        slope = (f(*plus) - f(*minus)) / 2e-3              # f is linear in each of the three: no error but rounding
        # the gradient's 2-norm bound times |v|
        assert abs(slope - float((grad.double() * v).sum())) <= 4 * 2.0 ** -16 * float(grad.double().norm() * v.norm())


def test_captured_replayed_and_beside_one_another(qb):
    # one graph serves other batches of the same buffers; two streams run at once with a workspace each
    size, n = (512, 1024, 4, 8, 64), 6
    bank = ra.make_bank(qb, n, *size, seed=9)
    T = 220
    cu, ids = torch.zeros(31, dtype=torch.int32, device=DEV), torch.zeros(30, dtype=torch.int32, device=DEV)
    X, Y, dY, dX = _randn(1, T, 512), _randn(2, T, 1024, dtype=torch.float32), _randn(3, T, 1024), _randn(4, T, 512, dtype=torch.float32)
    outs = torch.empty(T, dtype=torch.int32, device=DEV), torch.empty(n + 1, dtype=torch.int32, device=DEV)
    grads = torch.empty(bank.A.shape, device=DEV), torch.empty(bank.B.shape, device=DEV)
    ws, wsb = qb.alloc_adapters_workspace(bank, T), qb.alloc_adapters_workspace(bank, T, backward=True)
    Y0, dX0 = Y.clone(), dX.clone()

    def batch(seed):
        r = random.Random(seed)
        lens = [r.choice([1, 1, 1, 0, 5, 40]) for _ in range(30)]
        while sum(lens) > T:
            lens[lens.index(max(lens))] = 1
        c = [0]
        for k in lens:
            c.append(c[-1] + k)
        who = [r.randrange(-1, n) for _ in range(30)]
        cu.copy_(torch.tensor(c, dtype=torch.int32))
        ids.copy_(torch.tensor(who, dtype=torch.int32))
        return c, who

    def step():
        p = qb.adapter_plan(cu, ids, n, T, outs=outs)
        qb.adapters_fwd(bank, p, X, Y, ws=ws)
        qb.adapters_bwd(bank, p, X, dY, dX, outs=grads, ws=wsb)

    batch(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    side.synchronize()
    for seed in (1, 2, 3):
        c, who = batch(seed)
        Y.copy_(Y0)
        dX.copy_(dX0)
        graph.replay()
        torch.cuda.synchronize()
        want, bound = ra.ref_fwd(bank, c, who, X, Y0)
        ra.check(Y, want, bound, 2, 576, ("Y", torch.float32), Y0)
        want, bound = ra.ref_bwd(bank, c, who, X, dY, dX0)
        ra.check(dX, want[0], bound[0], 2, 1088, ("dX", torch.float32), dX0)
        ra.check(grads[0], want[1], bound[1], 4, 1500, ("dA", torch.float32))
        ra.check(grads[1], want[2], bound[2], 4, 1500, ("dB", torch.float32))
    plan = qb.adapter_plan(cu, ids, n, T)
    torch.cuda.synchronize()
    alone = qb.adapters_fwd(bank, plan, X, Y0.clone())
    results, streams = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(12):
        s = streams[k % 2]
        with torch.cuda.stream(s):
            y = Y0.clone()
        results.append(qb.adapters_fwd(bank, plan, X, y, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(alone, y) for y in results)


def test_rows_beyond_32_bits_of_elements(qb):
    # the last rows of buffers of more than 2^31 elements
    size = (512, 32768, 8, 8, 16)
    T = (1 << 31) // 32768 + 130
    bank = ra.make_bank(qb, 2, *size, seed=3)
    X, Y = torch.zeros(T, 512, dtype=torch.bfloat16, device=DEV), torch.zeros(T, 32768, dtype=torch.bfloat16, device=DEV)
    lens, ids = [T - 121, 1, 120], [-1, 1, 0]
    X[-121:] = _randn(1, 121, 512)
    cu, di, _ = ra.requests(lens, ids)
    plan = qb.adapter_plan(cu, di, 2, T)
    qb.adapters_fwd(bank, plan, X, Y)
    want, bound = ra.ref_fwd(bank, [0, 1, 121], [1, 0], X[-121:], torch.zeros(121, 32768, device=DEV))
    ra.check(Y[-121:], want, bound, 2, 528, ("Y", torch.bfloat16))
    assert not bool(Y[:-121].any())


def test_refusals(qb):
    bank, cu, ids, plan, T = _case(qb, (256, 256, 4, 4, 32), "tiles", 4)
    X, Y = _randn(1, T, 256), _randn(2, T, 256)
    for bad in (lambda: qb.adapters_fwd(bank, plan, X[:, :128], Y), lambda: qb.adapters_fwd(bank, plan, X.float(), Y),
                lambda: qb.adapters_fwd(bank, plan, X, Y.half()), lambda: qb.adapters_fwd(bank, plan, X, Y[:-1]),
                lambda: qb.adapters_fwd(bank, plan, X.T.contiguous().T, Y), lambda: qb.adapters_fwd(bank, plan, X, Y.cpu()),
                lambda: qb.adapters_fwd(bank, plan, X, Y[:1].expand(T, 256)),
                lambda: qb.adapters_fwd(bank, qb.AdapterPlan(plan.rows[:5], plan.start), X, Y),
                lambda: qb.adapters_fwd(bank, qb.AdapterPlan(plan.rows, plan.start[:3]), X, Y),
                lambda: qb.adapters_fwd(bank, qb.AdapterPlan(plan.rows.long(), plan.start), X, Y),
                lambda: qb.adapters_fwd(bank, plan, X, Y, ws=torch.empty(64, device=DEV)),
                lambda: qb.adapters_fwd(qb.AdapterBank(256, 256, 4, 4, bank.A, bank.B[:2], bank.scaling), plan, X, Y),
                lambda: qb.adapters_fwd(qb.AdapterBank(256, 256, 3, 4, bank.A, bank.B, bank.scaling), plan, X, Y),
                lambda: qb.adapters_bwd(bank, plan, X, Y, outs=(None, torch.empty(3, device=DEV)))):
        with pytest.raises(ValueError):
            bad()
    for status, bad in ((qb.ERR_WORKSPACE, lambda: qb.adapters_fwd(bank, plan, X, Y, ws=torch.empty(256, dtype=torch.uint8, device=DEV))),
                        (qb.ERR_INVALID_ARG, lambda: qb.adapters_fwd(bank, plan, X, X)),
                        (qb.ERR_INVALID_ARG, lambda: qb.adapters_bwd(bank, plan, None, Y)),
                        (qb.ERR_INVALID_ARG, lambda: qb.adapters_bwd(bank, plan, X, Y, Y)),
                        (qb.ERR_UNSUPPORTED, lambda: qb.adapter_plan(torch.zeros(8194, dtype=torch.int32, device=DEV),
                                                                     torch.zeros(8193, dtype=torch.int32, device=DEV), 3, 9)),
                        (qb.ERR_INVALID_ARG, lambda: qb.adapter_plan(plan.start, plan.start[:3], 3, 9, outs=(plan.rows, plan.start)))):
        with pytest.raises(qb.QbloraError) as e:
            bad()
        assert e.value.status == status
    # nothing to do
    empty = qb.adapters_fwd(bank, plan, X[:0], Y[:0])
    assert empty.shape == (0, 256)
    _, dA, dB = qb.adapters_bwd(bank, plan, X[:0], Y[:0])
    assert not bool(dA.any()) and not bool(dB.any())


@pytest.mark.parametrize("size", [(512, 256, 4, 4, 64), (1024, 1024, 8, 8, 256), (640, 1152, 2, 16, 136)], ids=str)
@pytest.mark.parametrize("lens,ids", [([513, 528, 512, 40, 1100], [0, 1, 2, 3, 5]), ([4100, 3, 530, 1025], [0, 1, 2, 3]), ([250, 300, 700, 7, 2400], [1, 1, 0, 2, 1])],
                         ids=["near the least", "one large", "in pieces"])
def test_gradients_of_many_rows(qb, size, lens, ids):
    # adapters whose rows are cut into parts, next to ones that are not, the last one's rows up to the end of the workspace
    n = 6
    bank = ra.make_bank(qb, n, *size, seed=21, ranks=[size[4], 5, size[4], size[4] // 2, 1, size[4]])
    cu, di, T = ra.requests(lens, ids)
    plan = qb.adapter_plan(cu, di, n, T)
    X, dY = _randn(3, T, size[0]), _randn(4, T, size[1])
    ws = qb.alloc_adapters_workspace(bank, T, backward=True)
    ws.fill_(0xff)                                           # whatever a call finds there
    nan = lambda t: torch.full(t.shape, float("nan"), device=DEV)  # noqa: E731
    _, dA, dB = qb.adapters_bwd(bank, plan, X, dY, outs=(nan(bank.A), nan(bank.B)), ws=ws)
    want, bound = ra.ref_bwd(bank, cu.tolist(), ids, X, dY, torch.zeros(T, size[0], device=DEV))
    ra.check(dA, want[1], bound[1], 4, size[1] + size[0] // size[2] + T, ("dA", torch.float32))
    ra.check(dB, want[2], bound[2], 4, size[0] + size[1] // size[3] + T, ("dB", torch.float32))
    for _ in range(3):
        again = qb.adapters_bwd(bank, plan, X, dY, ws=ws)
        assert torch.equal(again[1], dA) and torch.equal(again[2], dB)
    # the numbers of other adapters' rows change nothing
    lens2, ids2 = lens[:1] + [900], ids[:1] + [4]
    cu2, di2, T2 = ra.requests(lens2, ids2, T)
    other = qb.adapters_bwd(bank, qb.adapter_plan(cu2, di2, n, T), X, dY, ws=ws)
    if ids.count(ids[0]) == 1:
        assert torch.equal(other[1][ids[0]], dA[ids[0]]) and torch.equal(other[2][ids[0]], dB[ids[0]])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size,n,rows", [((5200, 2112, 4, 4, 136), 60, 1), ((5200, 2112, 4, 4, 136), 200, 1), ((1024, 4160, 1, 1, 512), 40, 3),
                                         ((2080, 1040, 5, 2, 40), 150, 2), ((8192, 640, 64, 1, 256), 16, 16), ((64, 64, 1, 1, 8), 4096, 0),
                                         ((128, 192, 2, 2, 16), 300, 4)],
                         ids=["60 of one", "200 of one", "rank 512", "lambda 5", "16 of 16", "4096 adapters", "300 of four"])
def test_forward_of_many_adapters(qb, size, n, rows, dtype):
    # as many adapters as make the clusters small, some left out, ranks of all kinds; both sides of the number of rows that changes the path
    r = random.Random(n)
    ids = r.sample(range(n), min(n, 250))
    lens = [rows + b % 3 if rows else 1 + b % 2 for b in range(len(ids))]
    bank = ra.make_bank(qb, n, *size, ranks=[r.choice([size[4], size[4], size[4] // 2 + 1, 1, 0]) for _ in range(n)], seed=n)
    cu, di, T = ra.requests(lens, ids)
    for T in (T, max(T, 520)):
        X, Y0 = _randn(1, T, size[0]), _randn(2, T, size[1], dtype=dtype)
        Y = qb.adapters_fwd(bank, qb.adapter_plan(cu, di, n, T), X, Y0.clone())
        want, bound = ra.ref_fwd(bank, cu.tolist(), ids, X, Y0)
        ra.check(Y, want, bound, 2, size[0] + size[4], ("Y", dtype), Y0)
        assert torch.equal(Y[int(cu[-1]):], Y0[int(cu[-1]):])


def test_backward_of_many_adapters(qb):
    n, size = 4096, (64, 64, 1, 1, 8)
    r = random.Random(3)
    ids = [r.randrange(n) for _ in range(500)]
    lens = [r.choice([0, 1, 1, 2, 9]) for _ in ids]
    bank = ra.make_bank(qb, n, *size, seed=5)
    cu, di, T = ra.requests(lens, ids)
    X, dY, dX0 = _randn(3, T, 64), _randn(4, T, 64), _randn(5, T, 64, dtype=torch.float32)
    dX, dA, dB = qb.adapters_bwd(bank, qb.adapter_plan(cu, di, n, T), X, dY, dX0.clone())
    want, bound = ra.ref_bwd(bank, cu.tolist(), ids, X, dY, dX0)
    for got, w, b, name, base in zip((dX, dA, dB), want, bound, ("dX", "dA", "dB"), (dX0, None, None)):
        ra.check(got, w, b, 4, 128 + T, (name, torch.float32), base)


@pytest.mark.parametrize("rank", [504, 520, 1024, 1400, 1416, 2000])
def test_large_ranks(qb, rank):
    # both sides of what the kernels' shared memory holds
    size, n = (256, 192, 2, 4, rank), 3
    bank = ra.make_bank(qb, n, *size, ranks=[rank, 5, rank - 9], seed=rank)
    cu, di, T = ra.requests([20, 3, 1, 30], [0, 1, -1, 2])
    X, Y0, dY, dX0 = _randn(1, T, 256), _randn(2, T, 192, dtype=torch.float32), _randn(3, T, 192), _randn(4, T, 256)
    plan = qb.adapter_plan(cu, di, n, T)
    want, bound = ra.ref_fwd(bank, cu.tolist(), [0, 1, -1, 2], X, Y0)
    ra.check(qb.adapters_fwd(bank, plan, X, Y0.clone()), want, bound, 2, 256 + rank, ("Y", torch.float32), Y0)
    want, bound = ra.ref_bwd(bank, cu.tolist(), [0, 1, -1, 2], X, dY, dX0)
    dX, dA, dB = qb.adapters_bwd(bank, plan, X, dY, dX0.clone())
    ra.check(dX, want[0], bound[0], 2, 192 + rank, ("dX", torch.bfloat16), dX0)
    ra.check(dA, want[1], bound[1], 4, 320 + T, ("dA", torch.float32))
    ra.check(dB, want[2], bound[2], 4, 448 + T, ("dB", torch.float32))


def test_gradients_side_by_side_in_one_buffer_and_a_large_workspace(qb):
    bank, cu, ids, plan, T = _case(qb, (512, 256, 4, 4, 64), "wide", 31)
    X, dY = _randn(1, T, 512), _randn(2, T, 256)
    ws = qb.alloc_adapters_workspace(bank, 5000, backward=True)      # for more rows than there are
    both = torch.full((bank.A.numel() + bank.B.numel() + 2,), 7.0, device=DEV)
    dA, dB = both[1:1 + bank.A.numel()].view(bank.A.shape), both[1 + bank.A.numel():-1].view(bank.B.shape)
    qb.adapters_bwd(bank, plan, X, dY, outs=(dA, dB), ws=ws)         # (one element further than 16 bytes: the general path)
    want, bound = ra.ref_bwd(bank, cu, ids, X, dY, torch.zeros(T, 512, device=DEV))
    ra.check(dA, want[1], bound[1], 4, 384 + T, ("dA", torch.float32))
    ra.check(dB, want[2], bound[2], 4, 576 + T, ("dB", torch.float32))
    assert both[0] == 7 and both[-1] == 7
    with pytest.raises(qb.QbloraError) as e:
        qb.adapters_bwd(bank, plan, X, dY, outs=(dA, both[5:5 + bank.B.numel()].view(bank.B.shape)), ws=ws)
    assert e.value.status == qb.ERR_INVALID_ARG
    # the fast path: the same buffer for gradients on 16 bytes, and the same workspace for fewer rows
    dA, dB = both[:bank.A.numel()].view(bank.A.shape), both[bank.A.numel():-2].view(bank.B.shape)
    qb.adapters_bwd(bank, plan, X, dY, outs=(dA, dB), ws=ws)
    ra.check(dA, want[1], bound[1], 4, 384 + T, ("dA", torch.float32))
    ra.check(dB, want[2], bound[2], 4, 576 + T, ("dB", torch.float32))
    assert both[-1] == 7
