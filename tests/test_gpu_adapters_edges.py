"""Many adapters over one weight on the GPU: values at the ends of their types, in every path."""
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


# few rows, many rows, any sizes
PATHS = ["rows", "tiles", "general"]


def _path(monkeypatch, path):
    """Rows of the step's buffers that send a call the given way."""
    if path == "general":
        monkeypatch.setenv("QBLORA_FORCE_GENERAL", "1")
    return 600 if path == "tiles" else 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("path", PATHS)
def test_ranks_at_the_ends_of_their_type(qb, monkeypatch, path, dtype):
    # ranks are clamped to 0 .. rank, whatever an int32 can say: the bits of the clamped ones
    least = _path(monkeypatch, path)
    size = (256, 512, 4, 8, 40)
    ranks = [2 ** 31 - 1, 2 ** 31 - 15, 2 ** 31 - 16, 2 ** 30, 41, 40, 16, 0, -1, -2 ** 31]
    n = len(ranks)
    bank = ra.make_bank(qb, n, *size, ranks=[40] * n, seed=5)
    lens = [7, 1, 5, 8, 6, 3, 2, 2, 4, 1]
    cu, di, T = ra.requests(lens, list(range(n)), max(sum(lens), least))
    plan = qb.adapter_plan(cu, di, n, T)
    X, dY, Y0, dX0 = _randn(1, T, 256), _randn(2, T, 512), _randn(3, T, 512, dtype=dtype), _randn(4, T, 256, dtype=dtype)

    def results(values):
        bank.ranks.copy_(torch.tensor(values, dtype=torch.int32))
        return qb.adapters_fwd(bank, plan, X, Y0.clone()), *qb.adapters_bwd(bank, plan, X, dY, dX0.clone())

    want = results([min(max(k, 0), 40) for k in ranks])
    for got, ref in zip(results(ranks), want):
        assert torch.equal(got, ref)
    Y, _, dA, dB = want
    assert not torch.equal(Y[:7], Y0[:7]) and torch.equal(Y[34:], Y0[34:])
    assert bool(dA[0].any()) and bool(dB[0].any()) and not bool(dA[7:].any()) and not bool(dB[7:].any())


def _one_sign(bank, seed):
    """A without a negative number, B with one sign per column: infinite products of them add up to an infinity, not to NaN."""
    bank.A.abs_()
    g = torch.Generator(device=DEV).manual_seed(seed)
    bank.B.abs_()
    bank.B.mul_((torch.randint(0, 2, (bank.B.shape[2],), generator=g, device=DEV) * 2 - 1).bfloat16())


def _same_kind(got, want, bound, pairs, terms, name, dtype):
    """Infinities of the formula's sign and NaN where it has them, and its numbers, elsewhere within the bound."""
    assert torch.equal(got.isnan(), want.isnan()), name
    odd = want.isinf()
    assert torch.equal(got.isinf(), odd) and torch.equal(got[odd].double(), want[odd]), name
    fine = torch.isfinite(want)
    ra.check(got[fine], want[fine], bound[fine], pairs, terms, (name, dtype))


#               d_in  d_out  l1 l2  r
INF_SIZES = [(256, 512, 4, 4, 64), (640, 256, 8, 8, 40), (128, 128, 1, 1, 24), (320, 272, 5, 2, 264), (4096, 512, 2, 4, 16)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("where", ["X", "A", "B", "dY", "s"])
@pytest.mark.parametrize("size", INF_SIZES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("path", PATHS)
def test_infinities_are_those_of_the_formula(qb, monkeypatch, path, size, where, dtype):
    # numbers travel as sums of parts, and an infinity has no second part
    least = _path(monkeypatch, path)
    lens, ids, n = [9, 1, 16, 30, 7], [2, 0, 1, 0, 3], 4
    bank = ra.make_bank(qb, n, *size, seed=8)
    _one_sign(bank, 9)
    cu, di, T = ra.requests(lens, ids, max(sum(lens) + 2, least))
    plan = qb.adapter_plan(cu, di, n, T)
    X, dY = _randn(1, T, size[0]), _randn(2, T, size[1])
    X[5, ::7] = 0
    Y0, dX0 = _randn(3, T, size[1], dtype=dtype), _randn(4, T, size[0], dtype=dtype)
    inf = float("inf")
    if where == "X":
        X[3, 17], X[12, size[0] - 1], X[40, 0], X[40, 64] = inf, -inf, inf, -inf          # the last: NaN where both are in one sum
    elif where == "dY":
        dY[3, 17], dY[12, size[1] - 1], dY[40, 0], dY[40, 64] = inf, -inf, inf, -inf
    elif where == "A":
        bank.A[0, 3, 5], bank.A[2, -1, -1] = inf, inf
    elif where == "B":
        bank.B[0, 3, 5], bank.B[2, -1, -1] = inf, -inf
    else:
        bank.scaling[1] = inf
    cu = cu.tolist()
    want, bound = ra.ref_fwd(bank, cu, ids, X, Y0)
    _same_kind(qb.adapters_fwd(bank, plan, X, Y0.clone()), want, bound, 2, size[0] + size[4], "Y", dtype)
    if where == "s":
        return                                               # in front of dv's sums or behind them it gives NaN or infinities
    want, bound = ra.ref_bwd(bank, cu, ids, X, dY, dX0)
    dX, dA, dB = qb.adapters_bwd(bank, plan, X, dY, dX0.clone())
    _same_kind(dX, want[0], bound[0], 2, size[1] + size[4], "dX", dtype)
    _same_kind(dA, want[1], bound[1], 4, size[1] + size[0] // size[2] + T, "dA", torch.float32)
    _same_kind(dB, want[2], bound[2], 4, size[0] + size[1] // size[3] + T, "dB", torch.float32)


@pytest.mark.parametrize("path", PATHS)
def test_entries_passed_over_beside_infinite_weights(qb, monkeypatch, path):
    # a row number out of range adds nothing to the gradients, whatever its adapter holds; the rows that fill up a tile neither
    least = _path(monkeypatch, path)
    bank = ra.make_bank(qb, 2, 256, 512, 4, 4, 32, seed=8)
    _one_sign(bank, 9)
    bank.A[1, 3, 5], bank.B[1, 7, 6] = float("inf"), -float("inf")
    cu, di, T = ra.requests([5, 20, 3], [0, 1, 0], max(30, least))
    plan = qb.adapter_plan(cu, di, 2, T)
    X, dY, Y0 = _randn(1, T, 256), _randn(2, T, 512), _randn(3, T, 512)
    rows = plan.rows.clone()
    rows[8 + 4], rows[8 + 17] = -3, T + 7                    # rows 9 and 22, of adapter 1
    holes = qb.AdapterPlan(rows, plan.start)
    ids = [0, 1, 1, 1, 0]                                    # what is left
    parts = [slice(0, 5), slice(5, 9), slice(10, 22), slice(23, 25), slice(25, 28)]
    X2, dY2 = torch.cat([X[p] for p in parts]), torch.cat([dY[p] for p in parts])
    cu2 = [0]
    for p in parts:
        cu2.append(cu2[-1] + p.stop - p.start)
    want, bound = ra.ref_bwd(bank, cu2, ids, X2, dY2, torch.zeros(X2.shape, device=DEV))
    _, dA, dB = qb.adapters_bwd(bank, holes, X, dY)
    _same_kind(dA, want[1], bound[1], 4, 512 + 64 + T, "dA", torch.float32)
    _same_kind(dB, want[2], bound[2], 4, 256 + 128 + T, "dB", torch.float32)
    Y = qb.adapters_fwd(bank, holes, X, Y0.clone())
    assert torch.equal(Y[[9, 22]], Y0[[9, 22]])


@pytest.mark.parametrize("where", ["X", "dY", "A"])
def test_infinities_where_gradients_are_cut(qb, where):
    # one adapter of many rows, whose gradients are formed in parts; the waits of a call of many such values do not run out
    size, lens, ids = (512, 256, 4, 4, 64), [2300, 40], [1, 0]
    bank = ra.make_bank(qb, 2, *size, seed=18)
    _one_sign(bank, 9)
    cu, di, T = ra.requests(lens, ids)
    plan = qb.adapter_plan(cu, di, 2, T)
    X, dY, dX0 = _randn(1, T, 512), _randn(2, T, 256), _randn(4, T, 512, dtype=torch.float32)
    if where == "A":
        bank.A[1, 70, 9] = float("inf")
    else:
        t = X if where == "X" else dY
        t[1000, 33], t[2000, 200] = float("inf"), -float("inf")
    ws = qb.alloc_adapters_workspace(bank, T, backward=True)
    want, bound = ra.ref_bwd(bank, cu.tolist(), ids, X, dY, dX0)
    got = qb.adapters_bwd(bank, plan, X, dY, dX0.clone(), ws=ws)
    for g, w, b, name in zip(got, want, bound, ("dX", "dA", "dB")):
        _same_kind(g, w, b, 4, 1024 + T, name, torch.float32)
    X[::3, ::5], dY[::2, ::7] = float("inf"), -float("inf")
    dX, dA, dB = qb.adapters_bwd(bank, plan, X, dY, dX0.clone(), ws=ws)
    assert not bool(torch.isfinite(dA).any()) and qb.device_status(ws) == qb.OK


def test_ranks_of_more_rows_than_a_grid_has(qb):
    # the general path takes any rank: here above 65535
    size, n = (12, 6, 2, 3, 65536 + 77), 2
    bank = ra.make_bank(qb, n, *size, seed=3)
    cu, di, T = ra.requests([3, 1, 2], [1, -1, 0])
    plan, cu = qb.adapter_plan(cu, di, n, T), cu.tolist()
    X, dY, Y0, dX0 = _randn(1, T, 12), _randn(2, T, 6), _randn(3, T, 6, dtype=torch.float32), _randn(4, T, 12, dtype=torch.float32)
    want, bound = ra.ref_fwd(bank, cu, [1, -1, 0], X, Y0)
    ra.check(qb.adapters_fwd(bank, plan, X, Y0.clone()), want, bound, 0, 12 + size[4], ("Y", torch.float32), Y0)
    want, bound = ra.ref_bwd(bank, cu, [1, -1, 0], X, dY, dX0)
    dX, dA, dB = qb.adapters_bwd(bank, plan, X, dY, dX0.clone())
    ra.check(dX, want[0], bound[0], 0, 6 + size[4], ("dX", torch.float32), dX0)
    ra.check(dA, want[1], bound[1], 0, 18 + T, ("dA", torch.float32))
    ra.check(dB, want[2], bound[2], 0, 18 + T, ("dB", torch.float32))


def test_tensors_of_another_device_than_the_current_one_are_refused(qb, monkeypatch):
    # kernels run on the current device, where another one's addresses would be nobody's
    bank = ra.make_bank(qb, 2, 256, 512, 4, 4, 32, seed=8)
    cu, di, T = ra.requests([5, 20, 3], [0, 1, 0])
    plan = qb.adapter_plan(cu, di, 2, T)
    X, Y, p = _randn(1, T, 256), _randn(2, T, 512), torch.zeros(10, device=DEV)
    opt = qb.AdamW([p], [p.clone()])
    calls = [lambda: qb.adapter_plan(cu, di, 2, T), lambda: qb.adapters_fwd(bank, plan, X, Y), lambda: qb.adapters_bwd(bank, plan, X, Y),
             lambda: qb.AdamW([p], [p.clone()]), lambda: opt.set_grads([p.clone()]), opt.step]
    for call in calls:
        call()
    torch.cuda.synchronize()
    monkeypatch.setattr(qb, "_current_device", lambda: DEV_OTHER)
    for call in calls:
        with pytest.raises(ValueError):
            call()
    monkeypatch.undo()
    # tensors that are not where the bank is
    for bad in (lambda: qb.adapters_fwd(bank, plan, X.cpu(), Y), lambda: qb.adapters_fwd(bank, plan, X, Y, ws=torch.empty(1 << 20, dtype=torch.uint8)),
                lambda: qb.adapters_fwd(bank, qb.AdapterPlan(plan.rows.cpu(), plan.start), X, Y), lambda: qb.adapter_plan(cu.cpu(), di, 2, T),
                lambda: qb.adapter_plan(cu, di.cpu(), 2, T), lambda: qb.adapters_bwd(bank, plan, X.cpu(), Y),
                lambda: qb.adapters_fwd(qb.AdapterBank(256, 512, 4, 4, bank.A, bank.B.cpu(), bank.scaling), plan, X, Y)):
        with pytest.raises(ValueError):
            bad()


DEV_OTHER = 1                                                # an index; no such device is touched


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows", [255, 256, 257, 511, 512, 513])
def test_one_adapter_on_either_side_of_the_border(qb, rows, dtype):
    # all rows of the step belong to one adapter: both sides of the number of rows that changes the forward path
    size = (1024, 1408, 4, 8, 128)
    bank = ra.make_bank(qb, 3, *size, seed=rows)
    cu, di, T = ra.requests([rows], [1])
    X, Y0 = _randn(1, T, size[0]), _randn(2, T, size[1], dtype=dtype)
    plan = qb.adapter_plan(cu, di, 3, T)
    Y = qb.adapters_fwd(bank, plan, X, Y0.clone())
    want, bound = ra.ref_fwd(bank, cu.tolist(), [1], X, Y0)
    ra.check(Y, want, bound, 2, size[0] + size[4], ("Y", dtype), Y0)
    assert torch.equal(Y, qb.adapters_fwd(bank, plan, X, Y0.clone()))
