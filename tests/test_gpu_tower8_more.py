"""GPU tests of the tower in 8 bits: what its backward pass makes of masked infinities, of
an input that its owner has used again, and of the path between blocks."""
import numpy as np
import pytest
import torch

from oracle import eight as E
from test_gpu_tower8 import _need_gpu, eighth, f64, near  # noqa: F401

pytestmark = pytest.mark.gpu


def gradients(t, x, dz):
    t.forward(x)
    t.backward(dz)
    torch.cuda.synchronize()
    return {k: v.clone() for k, v in t.grads.items()}


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_infinite_gradients_of_masked_units(rows):
    """Units that no row uses may have any weight behind them: the gradients are those of a
    tower whose weights there are 0."""
    from paper_2510_12494_amd.tower8 import EightTower
    g = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, 24, generator=g).bfloat16().cuda()
    dz = (100 * torch.randn(rows, 64, generator=g)).bfloat16().cuda()
    found = []
    for weight in (0.0, 3e38):
        t = EightTower(24, 64, 256, 2, rows, seed=8)
        for l in range(2):
            t.params[f"b.{l}"][128:] = -1e6                    # a block of 128 of their own
            t.params[f"W2.{l}"][:, 128:] = weight
        t.refresh()
        found.append(gradients(t, x, dz))
        assert not t.h[0][:, 128:].any() and t.h[0][:, :128].any()
    for k, want in found[0].items():
        assert torch.isfinite(found[1][k]).all() and torch.equal(found[1][k], want), k
