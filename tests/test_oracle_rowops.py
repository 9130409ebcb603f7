"""Pins of the float64 row operators (CPU): torch's float64 layer norm and its
autograd gradients, central differences, and the dropout's keying against a
scalar Philox written out here."""
import numpy as np
import pytest
import torch

from oracle import rowops as R


def _scalar_block(seed, step, tag, row, q):
    m = 0xFFFFFFFF
    c = [step & m, row & m, q, (1 << 31) + ((row >> 32) << 16) + tag]
    k = [seed & m, seed >> 32]
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & m, (a >> 32) ^ c[3] ^ k[1], a & m]
        k = [(k[0] + 0x9E3779B9) & m, (k[1] + 0xBB67AE85) & m]
    return [h for w in c for h in (w & 0xFFFF, w >> 16)]


@pytest.mark.parametrize("seed,step,tag,row", [(1, 0, 0, 0), (0xDEADBEEF12345678, 77, 3, 5),
                                                 (2**64 - 1, 2**32 - 1, 65535, 2**47 - 1), (9, 4, 1, 2**32 + 6)])
def test_numbers_are_the_halves_of_one_block_per_eight_columns(seed, step, tag, row):
    got = R.numbers(seed, step, tag, [row], 19)[0]
    want = sum((_scalar_block(seed, step, tag, row, q) for q in range(3)), [])[:19]
    assert got.tolist() == want


def test_keep_rate_and_mean():
    n = 1 << 20
    for p in (0.1, 0.25, 0.5):
        keep = R.keep_mask(p, 11, 3, 2, np.arange(1024), n // 1024)
        q = R.threshold(p) / 65536
        assert abs(keep.mean() - (1 - q)) < 5 * np.sqrt(q * (1 - q) / n)
        assert abs(R.scale(p) * (1 - q) - 1) < 1e-15          # the expectation is exact
    assert R.keep_mask(0.0, 1, 1, 1, [0], 64).all() and not R.keep_mask(1.0, 1, 1, 1, [0], 64).any()


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 64), (9, 333)])
def test_layer_norm_equals_torch_in_float64(rows, cols):
    rng = np.random.default_rng(rows * 1000 + cols)
    x, dy = rng.normal(size=(rows, cols)), rng.normal(size=(rows, cols))
    gamma, beta = 1 + 0.1 * rng.normal(size=cols), rng.normal(size=cols)
    tx, tg, tb = (torch.tensor(v, requires_grad=True) for v in (x, gamma, beta))
    ty = torch.nn.functional.layer_norm(tx, (cols,), tg, tb, 1e-5)
    ty.backward(torch.tensor(dy))
    y, stats = R.layer_norm(x, gamma, beta, 1e-5)
    dx, dgamma, dbeta = R.layer_norm_backward(x, stats, gamma, dy)
    for a, b in ((y, ty.detach()), (dx, tx.grad), (dgamma, tg.grad), (dbeta, tb.grad)):
        np.testing.assert_allclose(a, b.numpy(), rtol=1e-9, atol=1e-11)


def test_residual_gradients_against_differences():
    rng = np.random.default_rng(5)
    rows, cols, p, eps = 4, 13, 0.3, 1e-5
    x, r, wy, ws = (rng.normal(size=(rows, cols)) for _ in range(4))
    gamma, beta = 1 + 0.1 * rng.normal(size=cols), rng.normal(size=cols)
    keep = R.keep_mask(p, 3, 1, 0, np.arange(rows), cols)

    def loss(x, r, gamma, beta):
        s, y, _ = R.residual(x, r, p, keep, gamma, beta, eps)
        return (wy * y).sum() + (ws * s).sum()

    s, _, stats = R.residual(x, r, p, keep, gamma, beta, eps)
    dr, dx, dgamma, dbeta = R.residual_backward(s, stats, gamma, wy, ws, p, keep)
    args = [x, r, gamma, beta]
    for i, grad in enumerate((dx, dr, dgamma, dbeta)):
        for at in np.ndindex(*args[i].shape):
            d = []
            for sign in (1, -1):
                moved = [a.copy() for a in args]
                moved[i][at] += sign * 1e-5
                d.append(loss(*moved))
            # central difference at 1e-5: truncation below 1e-8, cancellation below 1e-9
            assert abs((d[0] - d[1]) / 2e-5 - grad[at]) < 1e-7
    assert (dx[~keep] == 0).all()
