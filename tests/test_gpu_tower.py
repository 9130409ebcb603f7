"""GPU tests of the residual tower: its gradients against float64 autograd on the
same masks, a batch in two halves, and the example end to end."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import rowops as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs an MI355X")


def _reference(t, x, dz, row0, step):
    """Embedding and gradients of tower t in float64 on the CPU."""
    P = {k: v.double().cpu().requires_grad_() for k, v in t.params.items()}
    ids = np.arange(row0, row0 + len(x))

    def drop(v, tag):
        k = torch.from_numpy(R.keep_mask(t.p, t.seed, step, tag, ids, v.shape[1]))
        return torch.where(k, v * R.scale(t.p), 0.0)

    def norm(s, l):
        return torch.nn.functional.layer_norm(s, (t.width,), P[f"gamma.{l}"], P[f"beta.{l}"], 1e-5)

    s = x.double().cpu() @ P["W_in"].T
    y = norm(s, 0)
    for l in range(t.blocks):
        a = drop(torch.relu(y @ P[f"W1.{l}"].T + P[f"b.{l}"]), 2 * l)
        s = s + drop(a @ P[f"W2.{l}"].T, 2 * l + 1)
        y = norm(s, l + 1)
    y.backward(dz.double().cpu())
    return y.detach(), {k: v.grad for k, v in P.items()}


@pytest.mark.parametrize("width,hidden,blocks,rows", [(64, 96, 2, 300), (40, 33, 1, 77), (256, 256, 3, 1500)])
def test_gradients_equal_float64_autograd(width, hidden, blocks, rows):
    """float32: products of up to 256 terms and sums over the rows, a few
    layers deep: within 1e-4 of the largest entry (the bound of the float32
    workloads), apart from ReLUs within rounding of zero, of which a handful
    may flip (each moves an entry by at most one row's share)."""
    from paper_2510_12494_amd.tower import ResidualTower
    t = ResidualTower(24, width, hidden, blocks, rows + 50, "f32", p=0.25, seed=5)
    g = torch.Generator().manual_seed(rows)
    x, dz = torch.randn(rows, 24, generator=g), torch.randn(rows, width, generator=g) / rows
    z = t.forward(x.cuda(), row0=900, step=4)
    want, grads = _reference(t, x, dz, 900, 4)
    assert (z.double().cpu() - want).abs().max() <= 1e-4 * want.abs().max()
    t.backward(dz.cuda())
    for k, v in grads.items():
        err = (t.grads[k].double().cpu() - v).abs().max() / v.abs().max()
        assert err <= 1e-4 + 4.0 / rows * 0.05, (k, float(err))


def test_a_sample_does_not_depend_on_its_batch():
    from paper_2510_12494_amd.tower import ResidualTower
    t = ResidualTower(16, 64, 64, 2, 512, "f32", p=0.3, seed=3)
    x = torch.randn(512, 16, generator=torch.Generator().manual_seed(1)).cuda()
    whole = t.forward(x, row0=100, step=9).clone()
    halves = torch.cat([t.forward(x[:200], row0=100, step=9).clone(), t.forward(x[200:], row0=300, step=9).clone()])
    assert (whole - halves).abs().max() <= 1e-4 * whole.abs().max()
    assert (whole - t.forward(x, row0=100, step=10)).abs().max() > 0.1         # another step, other masks
    one = t.forward(x[7:8], train=False).clone()
    assert (one - t.forward(x, train=False)[7:8]).abs().max() <= 1e-4 * one.abs().max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_example_learns(dtype, capsys):
    spec = importlib.util.spec_from_file_location("residual_towers", os.path.join(ROOT, "examples", "residual_towers.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, right = m.main(["--steps", "120", "--rows", "9000", "--batch", "2048", "--width", "128", "--blocks", "2",
                            "--dtype", dtype])
    assert abs(losses[0] - np.log(2)) < 1e-3                  # a zero head: the logit is 0
    assert np.mean(losses[-10:]) < 0.9 * losses[0]
    assert right >= 0.5
    assert "scored 64 samples" in capsys.readouterr().out


def test_refusals():
    from paper_2510_12494_amd.tower import ResidualTower
    t = ResidualTower(16, 32, 32, 1, 64, "f32")
    for bad in (torch.zeros(65, 16), torch.zeros(4, 15), torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(0, 16)):
        with pytest.raises(ValueError):
            t.forward(bad.cuda())


def test_backward_needs_the_training_forward_of_its_rows():
    from paper_2510_12494_amd.tower import ResidualTower
    t = ResidualTower(16, 32, 32, 1, 64, "f32")
    x = torch.randn(64, 16, generator=torch.Generator().manual_seed(1)).cuda()
    dz = torch.ones(64, 32, device="cuda")
    with pytest.raises(ValueError):
        t.backward(dz)                                        # no forward yet
    t.forward(x)
    for bad in (dz[:63], dz[:, :31], dz.cpu()):
        with pytest.raises(ValueError):
            t.backward(bad)
    t.backward(dz)
    t.forward(x[:1], train=False)                             # scoring takes the buffers
    with pytest.raises(ValueError):
        t.backward(dz)
    with pytest.raises(ValueError):
        ResidualTower(16, 32, 32, 1, 64, "f16")


def test_gradient_of_one_row_in_any_layout():
    """A single row's stride says nothing about its length."""
    from paper_2510_12494_amd.tower import ResidualTower
    t = ResidualTower(16, 32, 32, 1, 64, "f32")
    g = torch.Generator().manual_seed(2)
    x, dz = torch.randn(1, 16, generator=g).cuda(), torch.randn(32, 1, generator=g).cuda()
    t.forward(x)
    t.backward(dz.T)                                          # strides (1, 1)
    got = {k: v.clone() for k, v in t.grads.items()}
    t.backward(dz.T.reshape(-1).reshape(1, 32).clone())
    assert all(torch.equal(got[k], v) for k, v in t.grads.items())
    assert t.grads["gamma.0"].abs().max() > 0


def test_training_forwards_without_a_step_differ_in_their_masks():
    """Each takes the step after the last one's; scoring takes none."""
    from paper_2510_12494_amd.tower import ResidualTower
    x = torch.randn(40, 16, generator=torch.Generator().manual_seed(4)).cuda()
    named = ResidualTower(16, 64, 64, 1, 64, "f32", p=0.3, seed=8)
    want = [named.forward(x, step=i).clone() for i in range(3)]
    t = ResidualTower(16, 64, 64, 1, 64, "f32", p=0.3, seed=8)
    for i in range(2):
        assert torch.equal(t.forward(x), want[i])
        t.forward(x, train=False)
    assert (want[0] - want[1]).abs().max() > 0.1
    assert torch.equal(t.forward(x, step=0), want[0])         # named: that one, and the next counts from it
    assert torch.equal(t.forward(x), want[1])
    assert torch.equal(t.forward(x), want[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weight_gradients_are_float32_sums(dtype):
    """Not rounded to the tower's type on their way to the float32 masters: within
    a float32 sum's bound of the float64 product of the buffers they come from."""
    from paper_2510_12494_amd.tower import ResidualTower
    rows = 60
    tdt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    t = ResidualTower(24, 64, 96, 1, 64, dtype, p=0.2, seed=6)
    g = torch.Generator().manual_seed(7)
    wide = torch.randn(rows, 30, generator=g).cuda().to(tdt)
    x, dz = wide[:, 3:27], torch.randn(rows, 64, generator=g).cuda()
    t.forward(x, row0=5, step=2)
    t.backward(dz)
    for name, d, v in (("W_in", t.ds, x), ("W1.0", t.dh, t.y[0])):
        d, v = d[:rows].double(), v[:rows].double()
        assert t.grads[name].dtype == torch.float32
        err = (t.grads[name].double() - d.T @ v).abs()
        assert bool((err <= (rows + 2) * 2.0 ** -24 * (d.abs().T @ v.abs()) + 1e-30).all()), name
    for name in ("W_in", "W1.0", "W2.0"):
        w = t.grads[name]
        assert bool((w != w.bfloat16().float()).any()), name


def test_operand_copies_are_of_what_the_products_read():
    from paper_2510_12494_amd.tower import ResidualTower
    t = ResidualTower(16, 32, 32, 2, 64)
    assert set(t.copies) == {"W_in"} | {f"{k}.{l}" for k in ("W1", "W2", "b") for l in range(2)}


def _reference_of_the_same_relus(t, x, dz, row0, step):
    """_reference with the tower's operand copies (the weights as its products
    read them) and the ReLU pattern of its own forward."""
    P = {k: (t.copies[k] if k in t.copies else v).double().cpu().requires_grad_() for k, v in t.params.items()}
    ids = np.arange(row0, row0 + len(x))

    def drop(v, tag):
        k = torch.from_numpy(R.keep_mask(t.p, t.seed, step, tag, ids, v.shape[1]))
        return torch.where(k, v * R.scale(t.p), 0.0)

    def norm(s, l):
        return torch.nn.functional.layer_norm(s, (t.width,), P[f"gamma.{l}"], P[f"beta.{l}"], 1e-5)

    s = x.double().cpu() @ P["W_in"].T
    y = norm(s, 0)
    for l in range(t.blocks):
        on = (t.h[l][:len(x)] > 0).cpu()
        h = torch.where(on, y @ P[f"W1.{l}"].T + P[f"b.{l}"], 0.0)
        s = s + drop(drop(h, 2 * l) @ P[f"W2.{l}"].T, 2 * l + 1)
        y = norm(s, l + 1)
    y.backward(dz.double().cpu())
    return y.detach(), {k: v.grad for k, v in P.items()}


def _rel(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


# A stored bf16 value is off by at most 2^-9 of itself, so a stored tensor by at
# most 2^-9 of its L2 norm; norms, random products and joins hand a relative error
# on about as it is.  The longest path stores, in a block, y, the ReLU's input and
# output, a, the branch and s going forward and dbranch, dh (three times), dy and
# ds going back: 12, and two more at either end, all added up as if they agreed.
def _bf16_bound(blocks):
    return (12 * blocks + 4) * 2.0 ** -9


@pytest.mark.parametrize("width,hidden,blocks,rows", [(64, 96, 2, 300), (40, 33, 1, 77), (256, 256, 2, 1500)])
def test_bf16_gradients_equal_float64_autograd(width, hidden, blocks, rows):
    from paper_2510_12494_amd.tower import ResidualTower
    t = ResidualTower(24, width, hidden, blocks, rows + 50, "bf16", p=0.25, seed=5)
    g = torch.Generator().manual_seed(rows)
    x, dz = torch.randn(rows, 24, generator=g).bfloat16(), torch.randn(rows, width, generator=g) / rows
    for l in range(blocks + 1):                               # values that show a factor left out
        t.params[f"gamma.{l}"].copy_(1 + 0.3 * torch.randn(width, generator=g))
        t.params[f"beta.{l}"].copy_(0.3 * torch.randn(width, generator=g))
    z = t.forward(x.cuda(), row0=900, step=4)
    want, grads = _reference_of_the_same_relus(t, x, dz, 900, 4)
    assert _rel(z, want) <= _bf16_bound(blocks)
    t.backward(dz.cuda())
    for k, v in grads.items():
        assert _rel(t.grads[k], v) <= _bf16_bound(blocks), (k, _rel(t.grads[k], v))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_trained_towers_score_single_samples_as_batches(dtype):
    """Two towers and a linear head learn a linear teacher of both parties'
    features; held-out samples scored one by one give the batch's scores, and
    are right far more often than by chance."""
    from paper_2510_12494_amd.tower import ResidualTower
    tdt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    g = torch.Generator().manual_seed(12)
    x = torch.randn(2400, 20, generator=g)
    label = (x @ torch.randn(20, generator=g) > 0).float().cuda()
    xa, xb = x[:, :8].to("cuda", tdt), x[:, 8:].to("cuda", tdt)
    A, B = ResidualTower(8, 64, 64, 2, 2048, dtype, 0.1, 1), ResidualTower(12, 64, 64, 2, 2048, dtype, 0.1, 2)
    head = torch.zeros(128, device="cuda")
    for _ in range(150):
        z = torch.cat([A.forward(xa[:2000]), B.forward(xb[:2000])], 1).float()
        d = (torch.sigmoid(z @ head) - label[:2000]) / 2000
        dz = d[:, None] * head
        head -= 0.1 * (z.T @ d)
        for t, part in ((A, dz[:, :64]), (B, dz[:, 64:])):
            t.backward(part)
            t.sgd(0.1)

    def score(rows):
        return torch.cat([A.forward(xa[rows], train=False), B.forward(xb[rows], train=False)], 1).float() @ head

    batch = score(slice(2000, 2400))
    one = torch.cat([score(slice(i, i + 1)) for i in range(2000, 2400)])
    # a batch's products may add up in another order: each stored value may be rounded the other way
    assert _rel(one, batch.double().cpu()) <= (_bf16_bound(2) if dtype == "bf16" else 1e-4)
    right = float(((one > 0) == (label[2000:] > 0.5)).float().mean())
    assert right >= 0.7                                       # chance: 0.5, with a deviation of 0.025
