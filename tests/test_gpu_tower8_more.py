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


@pytest.mark.parametrize("d_in,width,hidden,rows", [(24, 64, 96, 300), (64, 64, 64, 1), (130, 64, 130, 77)])
def test_an_input_that_is_used_again_before_the_backward_pass(d_in, width, hidden, rows):
    from paper_2510_12494_amd.tower8 import EightTower
    t = EightTower(d_in, width, hidden, 1, rows + 30, seed=2)
    g = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, d_in, generator=g).bfloat16().cuda()
    dz = torch.randn(rows, width, generator=g).bfloat16().cuda()
    want = gradients(t, x, dz)
    t.forward(x)
    x.fill_(float("nan"))
    t.backward(dz)
    torch.cuda.synchronize()
    assert torch.isfinite(want["W_in"]).all() and all(torch.equal(t.grads[k], v) for k, v in want.items())


def test_what_a_matrix_in_8_bits_stands_for():
    """Every byte of values and of powers, to the last bit."""
    from paper_2510_12494_amd.tower8 import Eight
    m = Eight(255, 256, "cuda")
    m.data.copy_(torch.arange(256, dtype=torch.uint8).expand(255, 256))
    m.scale[:, :255] = torch.arange(255, dtype=torch.uint8, device="cuda")
    powers = np.broadcast_to(np.arange(-127, 128), (2, 255))
    want = E.dequantize(np.broadcast_to(E.e4m3_table(), (255, 256)), powers)
    assert np.array_equal(m.values(255, 250).cpu().numpy(), want[:, :250], equal_nan=True)
