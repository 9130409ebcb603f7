"""Pins of the float64 definitions in oracle/eight.py (CPU)."""
import numpy as np
import pytest
import torch

from oracle import eight as E


def test_e4m3_table_and_rounding_equal_torch():
    bits = torch.arange(256, dtype=torch.uint8)
    want = bits.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(E.e4m3_table(), want, equal_nan=True)
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.uniform(-448, 448, 20000), rng.normal(size=20000) * 0.01, [0.0, 448.0, -448.0]])
    x = x.astype(np.float32)
    assert np.array_equal(E.e4m3_round(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_e4m3_rounding_is_the_nearest_value_and_ties_are_even():
    table = E.e4m3_table()
    grid = np.sort(table[np.isfinite(table)])
    mid = (grid[1:] + grid[:-1]) / 2
    x = np.concatenate([grid, mid, mid + 1e-9, mid - 1e-9])
    got = E.e4m3_round(x)
    near = np.abs(x[:, None] - grid[None, :]).min(1)
    assert np.allclose(np.abs(got - x), near, rtol=0, atol=1e-12)
    even = {abs(v) for v, b in zip(table, range(256)) if b % 2 == 0 and np.isfinite(v)}
    assert all(abs(v) in even for v in E.e4m3_round(mid))


def test_powers_are_the_smallest_that_fit():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(40, 300)) * np.exp(rng.normal(size=(40, 1)) * 20)
    x[3], x[4, :5], x[5, 7], x[6, 9] = 0.0, 448.0, np.inf, np.nan
    x[7] = 1e-45
    x[8, :128] = 448.0 * 2.0 ** 7
    x[9, :128] = np.nextafter(448.0, 500.0)
    q, p = E.quantize(x)
    assert q.shape == (40, 384) and p.shape == (3, 40) and not q[:, 300:].any()
    v = E.dequantize(q, p)[:, :300]
    for b in range(3):
        blk = x[:, b * 128:(b + 1) * 128]
        top = np.where(np.isfinite(blk), np.abs(blk), 0).max(1)
        assert (top <= np.ldexp(448.0, p[b])).all()
        assert ((p[b] == -127) | (top > np.ldexp(448.0, p[b] - 1))).all()
    assert p[0, 8] == 7 and p[0, 9] == 1 and p[0, 3] == -127
    assert np.isnan(v[5, 7]) and np.isnan(v[6, 9]) and np.isfinite(np.delete(v[5], 7)).all()
    ok = np.isfinite(x)
    top = np.repeat(np.ldexp(448.0, p.T), 128, axis=1)[:, :300]
    # half a step of the value, or of the smallest one
    assert (np.abs(v - x)[ok] <= np.maximum(np.abs(x) * 2.0 ** -4, top * 2.0 ** -10 / 448)[ok]).all()


def _differences(f, a, h):
    g = np.zeros_like(a)
    for i in np.ndindex(a.shape):
        b = a.copy()
        b[i] += h
        up = f(b)
        b[i] -= 2 * h
        g[i] = (up - f(b)) / (2 * h)
    return g


def test_rms_gradients_against_differences():
    rng = np.random.default_rng(3)
    x, r, gamma, dy, dsx = (rng.normal(size=(3, 7)) for _ in range(5))
    gamma = gamma[0]

    def f(x=x, gamma=gamma):
        s, _, y = E.rms_forward(x, r, gamma, 1e-3)
        return (y * dy).sum() + (s * dsx).sum()

    s, k, _ = E.rms_forward(x, r, gamma, 1e-3)
    dx, dgamma = E.rms_backward(s, k, dy, dsx, gamma)
    assert np.allclose(dx, _differences(lambda v: f(x=v), x, 1e-5), atol=1e-8)
    assert np.allclose(dgamma, _differences(lambda v: f(gamma=v), gamma, 1e-5), atol=1e-8)


@pytest.mark.parametrize("gone", [False, True])
def test_softmax_gradients_against_differences(gone):
    rng = np.random.default_rng(4)
    x, w, bias = rng.normal(size=(5, 3)), rng.normal(size=(6, 3)), rng.normal(size=6)
    labels, dloss = np.array([0, 5, -1, 3, 6]), rng.uniform(0.5, 1.5, 5)
    if gone:
        bias[2] = -np.inf

    def f(x=x, w=w, bias=bias):
        return (E.softmax_loss(x, w, bias, labels)[0] * dloss).sum()

    loss, lse = E.softmax_loss(x, w, bias, labels)
    assert loss[2] == loss[4] == 0
    t = torch.nn.functional.cross_entropy(torch.from_numpy(x @ w.T + bias), torch.tensor([0, 5, 0, 3, 0]), reduction="none")
    assert np.allclose(loss[[0, 1, 3]], t.numpy()[[0, 1, 3]])
    G = E.softmax_grad(x, w, bias, labels, lse, dloss)
    assert np.allclose(G @ w, _differences(lambda v: f(x=v), x, 1e-5), atol=1e-8)
    assert np.allclose(G.T @ x, _differences(lambda v: f(w=v), w, 1e-5), atol=1e-8)
    keep = np.isfinite(bias)
    assert np.allclose(G.sum(0)[keep], _differences(lambda v: f(bias=np.where(keep, v, bias)), np.where(keep, bias, 0.0), 1e-5)[keep],
                       atol=1e-8)
    assert not G[:, ~keep].any()


def test_a_label_of_a_class_taken_out_and_a_row_without_classes():
    x, w = np.ones((2, 2)), np.ones((3, 2))
    loss, lse = E.softmax_loss(x, w, np.array([0.0, -np.inf, 0.0]), np.array([1, 0]))
    assert loss[0] == np.inf and np.isclose(loss[1], np.log(2.0))
    loss, lse = E.softmax_loss(x, w, np.full(3, -np.inf), np.array([1, -1]))
    assert loss[0] == np.inf and loss[1] == 0 and np.isneginf(lse).all()
    G = E.softmax_grad(x, w, np.full(3, -np.inf), np.array([1, -1]), lse, np.ones(2))
    assert not G.any()
