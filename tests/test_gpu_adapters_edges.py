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
