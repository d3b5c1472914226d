"""That the bound on fp32 results of the calls for many adapters tells two parts, or a product of parts left out, from three."""
import torch

from tests import _adapters_parts as rp


def test_two_parts_are_seen():
    g = torch.Generator().manual_seed(1)
    x, W = torch.randn(200, 1024, generator=g), torch.randn(1024, 300, generator=g).bfloat16().double()
    want = x.double() @ W
    assert rp.off(rp.split(x, 2) @ W, want) > 2 * rp.LIMIT
    assert rp.off(rp.split(x, 3) @ W, want) < rp.LIMIT / 64
    # a gradient: both sides in three parts, without the product of the first by the third
    y = torch.randn(200, 300, generator=g)
    want = x.double().T @ y.double()
    first, third = rp.split(x, 1), rp.split(y, 3) - rp.split(y, 2)
    full = rp.split(x, 3).T @ rp.split(y, 3)
    assert rp.off(full, want) < rp.LIMIT / 64 and rp.off(full - first.T @ third, want) > 2 * rp.LIMIT
