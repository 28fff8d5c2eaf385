"""GPU parity of the verification of drafted tokens where a batch is large enough for slices of 4096 and 8192 values and for more than
three launches ahead of the last one: choices equal to the oracle's."""
import pytest
import torch

from tests.test_gpu_drafts import Drafts, dev  # noqa: F401

pytestmark = pytest.mark.gpu


def slice_of(B, V):
    size = 8192
    while size > 2048 and B * -(-V // size) < 1024:
        size //= 2
    return size


@pytest.mark.parametrize("B,V,size", [(64, 66001, 4096), (64, 128001, 8192), (130, 33000, 4096), (260, 32769, 8192)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_slices(dev, B, V, size, dtype):
    # (five launches ahead of the last one at 64 requests of more than 65536 tokens, four at 130, five at 260)
    assert slice_of(B, V) == size
    new = [2 + i % 4 if B > 64 else 3 + i % 7 for i in range(B)]
    new[1], new[B // 2] = 0, 12
    d = Drafts(new, V, seed=V + B, dtype=dtype, noise=2.5, peak=1.5, width=12)
    assert d.run(dev) == d.want()
    assert d.run(dev, False) == d.want(False)


def test_large_slices_in_chains(dev):
    d = Drafts([5] * 64, 128001, seed=9, chain=True)
    assert d.run(dev) == d.want()
    assert d.run(dev, False) == d.want(False)
