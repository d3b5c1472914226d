"""Accuracy of the fp32 results of the calls for many adapters, on the fast paths: three parts, sums emptied every 256 terms."""
import pytest
import torch

from tests import _adapters as ra
from tests import _adapters_parts as rp
from tests._adapters import DEV

pytestmark = pytest.mark.gpu

#         d_in  d_out  l1  l2   r
SIZES = [(512, 256, 4, 4, 64), (4096, 2048, 64, 64, 16), (2048, 2048, 1, 1, 128), (4096, 1024, 2, 2, 256), (8192, 512, 4, 1, 48),
         (256, 4096, 2, 4, 512), (256, 192, 2, 4, 1024), (1024, 512, 8, 2, 1400)]


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_b200 import binding
    return binding


@pytest.mark.parametrize("lens,ids", [([1] * 20 + [9, 30], None), ([300, 1, 40, 259], [0, 1, 2, 0]), ([1900, 600], [0, 2])], ids=["few", "many", "cut"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_fp32_results_hold_three_parts(qb, size, lens, ids):
    n = 3
    ids = ids or [b % n for b in range(len(lens))]
    bank = ra.make_bank(qb, n, *size, seed=7)
    cu, di, T = ra.requests(lens, ids)
    g = torch.Generator(device=DEV).manual_seed(4)
    X, dY = (torch.randn(T, w, generator=g, device=DEV).bfloat16() for w in size[:2])
    plan, cu = qb.adapter_plan(cu, di, n, T), cu.tolist()
    Y0, dX0 = torch.zeros(T, size[1], device=DEV), torch.zeros(T, size[0], device=DEV)
    Y = qb.adapters_fwd(bank, plan, X, Y0.clone())
    dX, dA, dB = qb.adapters_bwd(bank, plan, X, dY, dX0.clone())
    want = [ra.ref_fwd(bank, cu, ids, X, Y0)[0], *ra.ref_bwd(bank, cu, ids, X, dY, dX0)[0]]
    got = {name: rp.off(x, w) for name, x, w in zip(("Y", "dX", "dA", "dB"), (Y, dX, dA, dB), want)}
    print(size, {k: f"{v / rp.LIMIT:.2f}" for k, v in got.items()})
    assert max(got.values()) <= rp.LIMIT, got
