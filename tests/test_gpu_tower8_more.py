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


class Recorded:
    """A tower's backward pass with what each of its norms and weight gradients read and wrote."""

    def __init__(self, t):
        self.norms, self.products, self.sums = {}, {}, []
        norm, grad, sums = t._norm_backward, t._weight_grad, t._column_sums

        def norm_backward(l, rows, dy, ds, dx, st):
            before = f64(dy[:rows]), None if ds is None else f64(ds[:rows])
            norm(l, rows, dy, ds, dx, st)
            self.norms[l] = (*before, f64(dx[:rows]))

        def weight_grad(d, x, name, st):
            self.products[name] = f64(d)
            grad(d, x, name, st)

        def column_sums(d, out, st):
            self.sums.append(f64(d))
            sums(d, out, st)

        t._norm_backward, t._weight_grad, t._column_sums = norm_backward, weight_grad, column_sums


@pytest.mark.parametrize("d_in,width,hidden,blocks,rows", [(24, 64, 96, 2, 300), (140, 256, 256, 3, 1500), (40, 130, 33, 2, 77),
                                                          (8, 128, 128, 4, 1)])
def test_the_backward_pass_through_every_block(d_in, width, hidden, blocks, rows):
    """Every gradient, and what each block hands to the one below it, against float64 on the
    operands that are stored: a value is off by its rounding, and 2^-12 of the largest for
    sums and products."""
    from paper_2510_12494_amd.tower8 import EightTower
    t = EightTower(d_in, width, hidden, blocks, rows + 20, seed=6)
    g = torch.Generator().manual_seed(rows + blocks)
    for l in range(blocks + 1):
        t.params[f"gamma.{l}"].copy_(1 + 0.3 * torch.randn(width, generator=g))
    for l in range(blocks):
        t.params[f"b.{l}"].copy_(0.3 * torch.randn(hidden, generator=g))
    x = torch.randn(rows, d_in, generator=g).bfloat16()
    dz = (torch.randn(rows, width, generator=g) * torch.exp(torch.randn(rows, 1, generator=g)) / rows).bfloat16()
    r = Recorded(t)
    t.forward(x.cuda())
    t.backward(dz.cuda())
    torch.cuda.synchronize()
    P, G = ({k: f64(v) for k, v in d.items()} for d in (t.params, t.grads))
    half = 2.0 ** -8
    assert sorted(r.norms) == list(range(blocks + 1)) and len(r.sums) == blocks
    assert np.array_equal(r.norms[blocks][0], f64(dz)) and r.norms[blocks][1] is None
    for l in range(blocks + 1):
        dy, ds, dx = r.norms[l]
        want, dgamma = E.rms_backward(f64(t.s[l][:rows]), f64(t.stats[l][:rows]), dy, 0.0 if ds is None else ds, P[f"gamma.{l}"])
        near(dx, want, half, f"ds_{l}")
        near(G[f"gamma.{l}"], dgamma, 0, f"dgamma.{l}")
    for l in reversed(range(blocks)):
        above, (dy, ds, _) = r.norms[l + 1][2], r.norms[l]
        h, y, dh = f64(t.h[l][:rows]), f64(t.y[l][:rows]), r.products[f"W1.{l}"]
        # the gradient of s_{l+1} goes into the branch and, as it is, past it
        assert np.array_equal(r.products[f"W2.{l}"], above) and np.array_equal(ds, above)
        near(G[f"W2.{l}"], eighth(above.T) @ eighth(h.T).T, 0, f"dW2.{l}")
        near(dh, np.where(h > 0, eighth(above) @ eighth(P[f"W2.{l}"].T).T, 0.0), half, f"dh_{l}")
        assert np.array_equal(r.sums[blocks - 1 - l], dh)
        near(G[f"b.{l}"], dh.sum(0), 0, f"db.{l}")
        near(G[f"W1.{l}"], eighth(dh.T) @ eighth(y.T).T, 0, f"dW1.{l}")
        near(dy, eighth(dh) @ eighth(P[f"W1.{l}"].T).T, half, f"dy_{l}")
    assert np.array_equal(r.products["W_in"], r.norms[0][2])
    near(G["W_in"], eighth(r.norms[0][2].T) @ eighth(f64(x).T).T, 0, "dW_in")


def test_an_update_reaches_the_copies_in_8_bits():
    from paper_2510_12494_amd.tower8 import EightTower
    t = EightTower(40, 130, 200, 2, 64, seed=3)
    g = torch.Generator().manual_seed(1)
    before = {k: v.clone() for k, v in t.params.items()}
    grads = gradients(t, torch.randn(50, 40, generator=g).bfloat16().cuda(), torch.randn(50, 130, generator=g).cuda())
    t.sgd(0.25)
    torch.cuda.synchronize()
    for k, v in t.params.items():
        assert torch.equal(v, before[k] - 0.25 * grads[k]) and float(grads[k].abs().max()) > 0
    for k, q in t.W.items():
        w = f64(t.params[k])
        assert not np.array_equal(w, f64(before[k]))
        for m, v in [(q, w)] + ([(t.WT[k], w.T)] if k in t.WT else []):
            assert np.array_equal(m.values(*v.shape).cpu().numpy(), eighth(np.ascontiguousarray(v)))
    assert sorted(t.W) == ["W1.0", "W1.1", "W2.0", "W2.1", "W_in"] and len(t.WT) == 4
