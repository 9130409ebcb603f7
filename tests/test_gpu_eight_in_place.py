"""GPU tests of calls that the header allows for the operators of towers in 8 bits: results
in the place of an input, and calls that run at the same time."""
import numpy as np
import pytest
import torch

from test_gpu_eight import EPS, Eight, Loss, Mat, V, _need_gpu, activations, gradients, matmul8, ptr, quantize, rms, vec  # noqa: F401

pytestmark = pytest.mark.gpu

SIZES = [(1, 7), (3, 1024), (300, 24), (2000, 130), (2500, 1030), (900, 2000), (700, 5001), (300, 8200), (40, 16390), (20, 32768)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("over", ["s", "dy", "ds"])
def test_rms_backward_in_place(V, dt, rows, cols, over):
    """dx over each input, with and without dgamma: the bits of dx elsewhere."""
    rng = np.random.default_rng(rows + cols)
    values = {k: f(rng, rows, cols) for k, f in (("s", activations), ("dy", gradients), ("ds", gradients))}
    stats, gamma = vec(rows, rng.uniform(0.5, 2, rows)), vec(cols, 1 + 0.1 * rng.normal(size=cols))
    size = V.vfl_norm_workspace_size(rows, cols)
    ws = torch.empty(size + 16, dtype=torch.uint8, device="cuda")
    for weights in (True, False):
        found = []
        for place in (None, over):
            m = {k: Mat(dt, rows, cols, cols + 3, 1, v) for k, v in values.items()}
            dx, dgamma = m[place] if place else Mat(dt, rows, cols, cols + 3, 1), vec(cols)
            a = V.vfl_rmsnorm_args()
            a.dtype, a.rows, a.cols, a.stats, a.gamma = V.VFL_BF16 if dt == "bf16" else V.VFL_F32, rows, cols, ptr(stats), ptr(gamma)
            for k, v in m.items():
                v.put(getattr(a, k))
            dx.put(a.dx)
            a.dgamma = ptr(dgamma) if weights else None
            a.workspace, a.workspace_bytes = ptr(ws), size
            V.vfl_rmsnorm_backward(a)
            torch.cuda.synchronize()
            found.append((dx.t.clone(), dgamma.clone()))
            for v in (*m.values(), dx):
                v.assert_guard()
        assert all(torch.equal(u, v) for u, v in zip(*found)) and bool(found[0][0].any())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rms_forward_in_place(V, dt, rows, cols):
    """s and y over x and r, either way."""
    rng = np.random.default_rng(rows * 3 + cols)
    xv, rv = activations(rng, rows, cols), activations(rng, rows, cols)
    gamma = vec(cols, 1 + 0.1 * rng.normal(size=cols))
    found = []
    for way in range(3):
        x, r = (Mat(dt, rows, cols, cols + 5, 2, v) for v in (xv, rv))
        s, y = ((x, r) if way == 1 else (r, x)) if way else (Mat(dt, rows, cols, cols + 5, 2) for _ in range(2))
        q, stats = Eight(rows, cols), vec(rows)
        rms(V, dt, rows, cols, x, r, gamma, s, y, q, stats)
        found.append((s.t.clone(), y.t.clone(), q._bytes().clone(), q._powers().clone(), stats.clone()))
        for m in (x, r, s, y, q):
            m.assert_guard()
    for other in found[1:]:
        assert all(torch.equal(u, v) for u, v in zip(found[0], other))


def test_calls_that_run_at_the_same_time(V):
    """Two streams with a workspace each, enqueued in turn: the results of one call alone."""
    losses = [Loss(V, dt, rows, dim, classes) for dt, rows, dim, classes in (("bf16", 600, 200, 9000), ("f32", 300, 130, 3000))]
    rng = np.random.default_rng(4)
    a, b = Eight(100, 20_000, 0, rng.normal(size=(100, 20_000))), Eight(200, 20_000, 0, rng.normal(size=(200, 20_000)))
    products = [Mat(dt, 100, 200) for dt in ("f32", "bf16")]
    room = [torch.empty(V.vfl_matmul8_workspace_size(100, 200, 20_000) + 16, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def both(streams):
        for _ in range(3):
            for i in range(2):
                matmul8(V, ("f32", "bf16")[i], a, b, products[i], 20_000, stream=streams[i], ws=room[i])
                losses[i].run(streams[i])
        torch.cuda.synchronize()
        return [t for i in range(2) for t in (products[i].t.clone(), *losses[i].results())]

    want = both((0, 0))
    side = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = both([s.cuda_stream for s in side])
        assert all(torch.equal(u, v) for u, v in zip(want, got))
    for t in losses:
        t.check()
