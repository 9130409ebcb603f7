"""GPU tests of the tower in 8 bits and of the head with many classes: every stage
against float64 on the operands that the stage read, a batch in parts, the
refusals, and the example."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import eight as E

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs an MI355X")


def f64(t):
    return t.double().cpu().numpy()


def eighth(t):
    """What a matrix stands for in 8 bits, in float64."""
    return E.dequantize(*E.quantize(t))[:, :t.shape[1]]


def near(got, want, half, what, also=0.0):
    """Within the rounding of a stored value (half a step), of a stored part of it
    (`also`: half a step of that), and what its float32 sums and 8-bit products lose: 2^-12
    of the largest value."""
    err = np.abs(got - want)
    ok = err <= half * np.abs(want) + 2.0 ** -8 * np.abs(also) + 2.0 ** -12 * np.abs(want).max() + 1e-30
    assert ok.all(), f"{what}: off by {err[~ok].max()}, the largest value is {np.abs(want).max()}"


@pytest.mark.parametrize("d_in,width,hidden,blocks,rows", [(24, 64, 96, 2, 300), (40, 130, 33, 1, 77), (140, 256, 256, 2, 1500),
                                                          (8, 128, 128, 1, 1)])
def test_every_stage_against_its_operands(d_in, width, hidden, blocks, rows):
    from paper_2510_12494_amd.tower8 import EightTower, EPS
    t = EightTower(d_in, width, hidden, blocks, rows + 50, seed=5)
    g = torch.Generator().manual_seed(rows)
    for l in range(blocks + 1):
        t.params[f"gamma.{l}"].copy_(1 + 0.3 * torch.randn(width, generator=g))
    for l in range(blocks):
        t.params[f"b.{l}"].copy_(0.3 * torch.randn(hidden, generator=g))
    x = torch.randn(rows, d_in, generator=g).bfloat16()
    dz = (torch.randn(rows, width, generator=g) * torch.exp(torch.randn(rows, 1, generator=g)) / rows).bfloat16()
    z = t.forward(x.cuda())
    P = {k: f64(v) for k, v in t.params.items()}
    half = 2.0 ** -8
    xd = f64(x)
    near(f64(t.s[0][:rows]), eighth(xd) @ eighth(P["W_in"]).T, half, "s_0")
    for l in range(blocks + 1):
        s = f64(t.s[l][:rows])
        k = E.rms_stats(s, EPS)
        if l:                     # of the float32 join, before it is rounded: k is off by half a step of s
            near(f64(t.stats[l][:rows]), k, half, "k")
            k = f64(t.stats[l][:rows])
        near(f64(t.y[l][:rows]), s * k[:, None] * P[f"gamma.{l}"], 2 * half, f"y_{l}")
    assert torch.equal(z, t.y[blocks][:rows])
    for l in range(blocks):
        # y in 8 bits comes from its float32 value, whose rounding to bf16 may move it a step of 2^-3
        h, y, s = f64(t.h[l][:rows]), f64(t.y[l][:rows]), f64(t.s[l][:rows])
        y32 = (s.astype(np.float32) * f64(t.stats[l][:rows]).astype(np.float32)[:, None] *
               P[f"gamma.{l}"].astype(np.float32)).astype(np.float64)
        if l == 0:                # s is the float32 value there is
            near(h, np.maximum(eighth(y32) @ eighth(P[f"W1.{l}"]).T + P[f"b.{l}"], 0), half, f"h_{l}")
        branch = eighth(h) @ eighth(P[f"W2.{l}"]).T            # stored before it is added
        near(f64(t.s[l + 1][:rows]), s + branch, half, f"s_{l + 1}", branch)

    t.backward(dz.cuda())
    G = {k: f64(v) for k, v in t.grads.items()}
    # the last block's gradients, from the tower's own buffers
    l = blocks - 1
    s, k = f64(t.s[blocks][:rows]), f64(t.stats[blocks][:rows])
    ds, dgamma = E.rms_backward(s, k, f64(dz), 0.0, P[f"gamma.{blocks}"])
    near(G[f"gamma.{blocks}"], dgamma, 0, "dgamma")
    h, y = f64(t.h[l][:rows]), f64(t.y[l][:rows])
    ds = f64(torch.from_numpy(ds).bfloat16())
    if blocks == 1:
        # stored gradients of the block: dh (masked) and dy, and the weights' from them
        dh = f64(t.dh[:rows])
        near(dh, np.where(h > 0, eighth(ds) @ eighth(P["W2.0"].T).T, 0.0), 2 * half, "dh")
        near(G["b.0"], dh.sum(0), 0, "db")
        near(f64(t.dy[:rows]), eighth(dh) @ eighth(P["W1.0"].T).T, half, "dy")
        near(G["W1.0"], eighth(dh.T) @ eighth(y.T).T, 0, "dW1")
        ds0, _ = E.rms_backward(f64(t.s[0][:rows]), f64(t.stats[0][:rows]), f64(t.dy[:rows]), ds, P["gamma.0"])
        near(f64(t.ds[1][:rows]), ds0, 2 * half, "ds_0")
        near(G["W_in"], eighth(f64(t.ds[1][:rows]).T) @ eighth(xd.T).T, 0, "dW_in")
    # ds is rounded from a float32 value: a handful of its entries may round the other way
    got, want = G[f"W2.{l}"], eighth(ds.T) @ eighth(h.T).T
    assert np.linalg.norm(got - want) <= 2.0 ** -8 * np.linalg.norm(want)


def test_a_sample_does_not_depend_on_its_batch():
    """Blocks of 8-bit values lie along a sample's own columns, and a norm's statistics
    do not depend on the batch; products may add up in another order."""
    from paper_2510_12494_amd.tower8 import EightTower
    t = EightTower(48, 128, 256, 2, 512, seed=3)
    x = torch.randn(512, 48, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    whole = t.forward(x).float().clone()
    halves = torch.cat([t.forward(x[:200]).float().clone(), t.forward(x[200:]).float().clone()])
    one = t.forward(x[7:8], train=False).float().clone()
    for got, want in ((halves, whole), (one, whole[7:8])):
        assert float((got - want).norm() / want.norm()) <= 2.0 ** -6


def test_refusals():
    from paper_2510_12494_amd.tower8 import ClassHead, EightTower
    t, head = EightTower(16, 64, 64, 1, 32), ClassHead(64, 10, 32)
    x = torch.zeros(8, 16, dtype=torch.bfloat16, device="cuda")
    z, lab = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    for bad in (x.float(), x[:, :15], x[:0], torch.zeros(33, 16, dtype=torch.bfloat16, device="cuda"), x.cpu(), x.T):
        with pytest.raises(ValueError):
            t.forward(bad)
    with pytest.raises(ValueError):
        t.backward(torch.zeros(8, 64, device="cuda"))          # no training forward yet
    t.forward(x, train=False)
    with pytest.raises(ValueError):
        t.backward(torch.zeros(8, 64, device="cuda"))
    t.forward(x)
    with pytest.raises(ValueError):
        t.backward(torch.zeros(7, 64, device="cuda"))
    for args in ((z.float(), lab), (z[:, :63], lab), (z, lab.long()), (z, lab[:7]), (z, lab.cpu())):
        with pytest.raises(ValueError):
            head.loss(*args)


def test_rows_that_are_one_row():
    """An expanded row's stride of 0 is not a matrix of that many rows."""
    from paper_2510_12494_amd.tower8 import ClassHead, EightTower
    t, head = EightTower(16, 64, 64, 1, 32), ClassHead(64, 10, 32)
    one = torch.zeros(1, 64, dtype=torch.bfloat16, device="cuda")
    lab = torch.zeros(8, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        t.forward(one[:, :16].expand(8, 16))
    with pytest.raises(ValueError):
        head.loss(one.expand(8, 64), lab)
    with pytest.raises(ValueError):
        t.forward(torch.as_strided(torch.zeros(256, dtype=torch.bfloat16, device="cuda"), (8, 16), (8, 1)))


def test_a_captured_step_is_the_eager_one():
    """Forward, head and backward in a graph, replayed between eager steps of other
    sizes, which use the same workspaces."""
    from paper_2510_12494_amd.tower8 import ClassHead, EightTower
    t, head = EightTower(40, 128, 320, 2, 3000, seed=6), ClassHead(128, 500, 3000, seed=7)
    g = torch.Generator().manual_seed(9)
    x = torch.zeros(2000, 40, dtype=torch.bfloat16, device="cuda")
    lab = torch.zeros(2000, dtype=torch.int32, device="cuda")

    def step(n):
        loss, dz = head.loss(t.forward(x[:n]), lab[:n])
        t.backward(dz)
        return loss

    def results(n):
        torch.cuda.synchronize()
        return [head.losses[:n].clone(), head.dW.clone(), head.dbias.clone()] + [v.clone() for v in t.grads.values()]

    step(2000)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(2000)
    for i in range(4):
        x.copy_(torch.randn(2000, 40, generator=g))
        lab.copy_(torch.randint(0, 500, (2000,), generator=g))
        step(2000)
        want = results(2000)
        step(77 + 300 * i)
        for v in t.grads.values():
            v.zero_()
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, results(2000)))
        assert float(want[0].sum()) > 0 and all(float(v.abs().sum()) > 0 for v in want)


def test_example_runs_and_learns_its_items(capsys):
    spec = importlib.util.spec_from_file_location("eight_bit_towers", os.path.join(ROOT, "examples", "eight_bit_towers.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, one = m.main(["--steps", "30", "--classes", "300", "--batch", "1024", "--width", "128", "--blocks", "1"])
    assert np.isfinite(losses).all() and np.isfinite(one) and len(losses) == 30
    assert "scored" in capsys.readouterr().out


def test_head_gradients_are_those_of_the_mean_loss():
    from paper_2510_12494_amd.tower8 import ClassHead
    rows, dim, classes = 200, 64, 900
    head = ClassHead(dim, classes, 256, seed=4)
    g = torch.Generator().manual_seed(2)
    z = torch.randn(rows, dim, generator=g).bfloat16()
    lab = torch.randint(-1, classes, (rows,), generator=g, dtype=torch.int32)
    head.bias.copy_(torch.randn(classes, generator=g))
    loss, dz = head.loss(z.cuda(), lab.cuda())
    w = head.copy.double().cpu().requires_grad_()
    b, zz = head.bias.double().cpu().requires_grad_(), z.double().requires_grad_()
    has = lab >= 0
    want = torch.nn.functional.cross_entropy((zz @ w.T + b)[has], lab[has].long(), reduction="none")
    (want.sum() / rows).backward()
    rel = lambda a, c: float((a.double().cpu() - c).norm() / c.norm())  # noqa: E731
    assert rel(loss[has.cuda()], want.detach()) <= 2.0 ** -18
    # G and the result are rounded to bf16, half a step (2^-8) each
    assert rel(dz, zz.grad) <= 2.0 ** -7 and rel(head.dW, w.grad) <= 2.0 ** -7 and rel(head.dbias, b.grad) <= 2.0 ** -16
    before = head.W.clone()
    head.sgd(0.5)
    assert torch.allclose(head.W, before - 0.5 * head.dW.float()) and torch.equal(head.copy, head.W.bfloat16())
