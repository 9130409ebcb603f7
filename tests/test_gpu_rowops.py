"""GPU tests of the row operators (dropout, layer norm, residual join) against
their float64 definitions in oracle/rowops.py.

Tolerances are bounds of float32 arithmetic (u = 2^-24), computed element by
element from the float64 values and fixed before the first run:
* a sum over a row passes at most SUM = 96 roundings per term (a thread's own
  terms, a wavefront's tree, the workgroup's wavefronts), a sum over rows at
  most min(rows, 512) + 32;
* every other operation adds its own rounding;
* a stored value must be the rounding of a value within the float32 bound:
  rounding is monotone, so it lies between the roundings of the bound's ends;
* first-order bounds are multiplied by 1.1 for the terms of second order, and
  the relative error of var + eps is required to stay below 0.1, where that
  holds.
Dropped elements are compared for equality: exactly zero, at the oracle's
places.
"""
import numpy as np
import pytest
import torch

from oracle import rowops as R

pytestmark = pytest.mark.gpu

U, SUM, SLACK = 2.0 ** -24, 96, 1.1
EPS = 1e-5
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
KEY = dict(seed=0x123456789ABCDEF, step=21, tag=3, row0=1000)


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs an MI355X")


@pytest.fixture(scope="module")
def V():
    from paper_2510_12494_amd import vfl
    return vfl


def rounded(a, dt):
    """Float64 values as they are stored (float32 bounds cover their own)."""
    if dt == "f32":
        return a
    # float64 -> float32 would round twice: to bf16 by the float64's own bits
    m, e = np.frexp(a)
    return np.ldexp(np.rint(m * 256.0), e - 8)


class Mat:
    """A [rows x cols] device matrix inside a guarded buffer: `lead` elements
    before its first one, ld from row to row."""

    GUARD = 77.0

    def __init__(self, dt, rows, cols, ld=0, lead=0, values=None):
        self.rows, self.cols, self.ld, self.lead = rows, cols, ld or cols, lead
        self.buf = torch.full((lead + rows * self.ld + 64,), self.GUARD, dtype=DT[dt], device="cuda")
        self.t = self.buf[lead:lead + rows * self.ld].view(rows, self.ld)[:, :cols]
        if values is not None:
            self.t.copy_(torch.from_numpy(np.asarray(values, np.float64)))

    def np(self):
        return self.t.double().cpu().numpy()

    def put(self, m):
        m.data, m.ld = self.t.data_ptr(), self.ld

    def assert_guard(self):
        """Nothing outside the matrix was written."""
        b = self.buf.clone()
        if self.rows:
            b[self.lead:self.lead + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = self.GUARD
        assert bool((b == self.GUARD).all())


def f32(n, values=None):
    t = torch.full((n + 8,), Mat.GUARD, dtype=torch.float32, device="cuda")
    if values is not None:
        t[:n] = torch.from_numpy(np.asarray(values)).float()
    return t


def stored(t, n):
    assert bool((t[n:] == Mat.GUARD).all())
    return t[:n].double().cpu().numpy()


def key(d, p, **kw):
    k = {**KEY, **kw}
    d.p, d.seed, d.step, d.tag, d.row0 = p, k["seed"], k["step"], k["tag"], k["row0"]


def keep(p, rows, cols, **kw):
    k = {**KEY, **kw}
    return R.keep_mask(p, k["seed"], k["step"], k["tag"], np.arange(k["row0"], k["row0"] + rows), cols)


def close(got, want, bound, what, dt="f32"):
    err = np.abs(got - want)
    bad = ~((got >= rounded(want - bound, dt)) & (got <= rounded(want + bound, dt)))
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} elements past their bound, worst "
                           f"{np.nanmax(np.where(bad, err / np.maximum(bound, 1e-300), 0)):.3g} times it, first at "
                           f"{np.argwhere(bad)[0]}")


def activations(rng, rows, cols):
    a = rng.normal(size=(rows, cols)) * np.exp(0.5 * rng.normal(size=cols)) + 0.5 * rng.normal(size=(rows, 1))
    if rows > 4:
        a[rows // 2] = 0.0                       # padding: no variance
    return a


# ------------------------------------------------------------------- bounds
def norm_bounds(v, ev, gamma, beta):
    """Errors of (y, stats) for row values v known to ev."""
    mean = v.mean(1, keepdims=True)
    d = v - mean
    var = (d * d).mean(1, keepdims=True)
    e_mean = SUM * U * np.abs(v).mean(1, keepdims=True) + ev.mean(1, keepdims=True) + 2 * U * np.abs(mean)
    e_d = ev + e_mean + U * np.abs(d)
    e_var = (2 * np.abs(d) * e_d + e_d * e_d).mean(1, keepdims=True) + (SUM + 4) * U * var
    assert (e_var < 0.1 * (var + EPS)).all()
    k = 1.0 / np.sqrt(var + EPS)
    rel = 0.5 * e_var / (var + EPS) * 1.2 + 4 * U
    h = d * k
    e_y = np.abs(gamma) * (k * e_d + np.abs(h) * (rel + 3 * U)) + 3 * U * (np.abs(h * gamma) + np.abs(beta))
    return SLACK * e_y, SLACK * np.concatenate([e_mean, k * rel], 1)


def grad_bounds(v, stats, gamma, dy):
    """Errors of the layer norm's (dx, dgamma, dbeta) before dx is stored."""
    mean, k = stats[:, :1], stats[:, 1:]
    h = (v - mean) * k
    g = dy * gamma
    e_h, e_g = 3 * U * np.abs(h), U * np.abs(g)
    mg, mgh = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    avg = lambda a: np.abs(a).mean(1, keepdims=True)  # noqa: E731
    e_mg = (SUM + 3) * U * avg(g) + 2 * U * np.abs(mg)
    e_mgh = (SUM + 6) * U * avg(g * h) + 2 * U * np.abs(mgh)
    dx = k * (g - mg - h * mgh)
    e_dx = k * (e_g + e_mg + np.abs(h) * e_mgh + e_h * np.abs(mgh)
                + 4 * U * (np.abs(g) + np.abs(mg) + np.abs(h * mgh))) + 2 * U * np.abs(dx)
    chain = min(len(v), 512) + 32
    e_dg = (np.abs(dy) * e_h).sum(0) + (chain + 1) * U * np.abs(dy * h).sum(0)
    e_db = chain * U * np.abs(dy).sum(0)
    return SLACK * e_dx, SLACK * e_dg + 1e-37, SLACK * e_db + 1e-37


# ------------------------------------------------------------------ dropout
# widths that end inside a chunk of eight, of a wavefront, of a workgroup;
# row strides and first elements of every alignment; one row and none
DROP_SHAPES = [(1, 1, 0, 0), (1, 7, 0, 1), (3, 8, 8, 0), (257, 9, 16, 3), (64, 333, 0, 0), (31, 333, 340, 5),
               (5, 1024, 0, 0), (130, 64, 72, 0), (2, 40001, 0, 1), (3001, 33, 0, 0), (0, 16, 0, 0), (77, 520, 521, 2)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,ld,lead", DROP_SHAPES)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(V, dt, rows, cols, ld, lead, p):
    rng = np.random.default_rng(rows * 7919 + cols)
    x = Mat(dt, rows, cols, ld, lead, activations(rng, rows, cols))
    y = Mat(dt, rows, cols, cols + lead, 0)      # another stride than x's
    a = V.vfl_dropout_args()
    a.dtype, a.rows, a.cols = (V.VFL_F32, V.VFL_BF16)[dt == "bf16"], rows, cols
    key(a.drop, p)
    x.put(a.x)
    y.put(a.y)
    V.vfl_dropout(a)
    want_keep = keep(p, rows, cols)
    got, xs = y.np(), x.np()
    want = R.dropout(xs, p, want_keep)
    assert (got[~want_keep] == 0).all()
    close(got, want, 2.5 * U * np.abs(want), "y", dt)
    if p == 0.0:
        assert (got == xs).all()
    y.assert_guard()
    x.assert_guard()
    # in place, the same bits
    x.put(a.y)
    V.vfl_dropout(a)
    assert torch.equal(x.t, y.t)
    x.assert_guard()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_dropped_elements_are_zero_whatever_their_value(V, dt):
    rows, cols, p = 16, 200, 0.5
    k = keep(p, rows, cols)
    vals = np.array([np.nan, np.inf, -np.inf, 3.0e38])[np.arange(rows * cols).reshape(rows, cols) % 4]
    x, y = Mat(dt, rows, cols, values=vals), Mat(dt, rows, cols)
    a = V.vfl_dropout_args()
    a.dtype, a.rows, a.cols = (V.VFL_F32, V.VFL_BF16)[dt == "bf16"], rows, cols
    key(a.drop, p)
    x.put(a.x)
    y.put(a.y)
    V.vfl_dropout(a)
    got, xs = y.np(), x.np()
    assert (got[~k] == 0).all()
    assert np.isnan(got[k & np.isnan(xs)]).all()
    assert (got[k & np.isinf(xs)] == xs[k & np.isinf(xs)]).all()


def test_masks_follow_the_sample_ids(V):
    """Rows keep their masks however a batch is split; another step, tag or
    seed gives another mask; ids past 2^32 use both words."""
    rows, cols, p = 96, 100, 0.4
    ones = np.ones((rows, cols))

    def mask(first, n, **kw):
        x, y = Mat("f32", n, cols, values=ones[:n]), Mat("f32", n, cols)
        a = V.vfl_dropout_args()
        a.dtype, a.rows, a.cols = V.VFL_F32, n, cols
        key(a.drop, p, **{**kw, "row0": kw.get("row0", KEY["row0"]) + first})
        x.put(a.x)
        y.put(a.y)
        V.vfl_dropout(a)
        return y.np() != 0

    whole = mask(0, rows)
    assert (np.concatenate([mask(0, 31), mask(31, 1), mask(32, 64)]) == whole).all()
    seen = [whole]
    for kw in ({"step": 22}, {"tag": 4}, {"seed": KEY["seed"] + 1}, {"seed": KEY["seed"] ^ 1 << 40},
               {"row0": KEY["row0"] + (1 << 32)}, {"row0": (1 << 47) - rows}, {"row0": (1 << 32) - 40}):
        m = mask(0, rows, **kw)
        assert (m == keep(p, rows, cols, **kw)).all()
        assert all((m != s).any() for s in seen)
        seen.append(m)


def test_step_on_the_device_in_a_replayed_graph(V):
    rows, cols, p = 50, 72, 0.3
    x, y = Mat("f32", rows, cols, values=np.ones((rows, cols))), Mat("f32", rows, cols)
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    a = V.vfl_dropout_args()
    a.dtype, a.rows, a.cols = V.VFL_F32, rows, cols
    key(a.drop, p)
    a.drop.step_dev = step.data_ptr()
    x.put(a.x)
    y.put(a.y)
    V.vfl_dropout(a, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        V.vfl_dropout(a, torch.cuda.current_stream().cuda_stream)
        step.add_(1)
    for i in range(4):
        g.replay()
        torch.cuda.synchronize()
        assert ((y.np() != 0) == keep(p, rows, cols, step=KEY["step"] + i)).all()
        y.t.zero_()


# --------------------------------------------------- layer norm and residual
# widths up to one wavefront's, several wavefronts', the limit, each with a
# part of a chunk; rows that leave row groups, workgroups and parts incomplete
SHAPES = [(1, 1, 0, 0), (3, 2, 0, 1), (5, 7, 9, 0), (130, 8, 0, 0), (67, 16, 0, 0), (1000, 13, 0, 0), (33, 63, 64, 1),
          (9000, 64, 0, 0), (300, 100, 104, 0), (37, 128, 0, 0), (129, 257, 0, 3), (40, 512, 0, 0), (2100, 500, 504, 0),
          (21, 1000, 0, 0), (1, 1024, 0, 0), (18, 1024, 1032, 8), (530, 1025, 0, 0), (7, 2048, 0, 0), (13, 2056, 0, 1),
          (11, 4096, 0, 0), (300, 4099, 0, 0), (6, 8192, 0, 0), (5, 8200, 8201, 0), (4, 16384, 0, 0), (3, 20001, 0, 1),
          (2, 32768, 0, 0), (1, 32767, 0, 0)]
DTS = ["f32", "bf16"]


class Call:
    """One layer's descriptor and its buffers."""

    def __init__(self, V, kind, dt, rows, cols, ld=0, lead=0, p=0.0, affine=True, rng=None):
        self.V, self.kind, self.dt, self.rows, self.cols, self.p = V, kind, dt, rows, cols, p
        rng = rng or np.random.default_rng(rows * 104729 + cols)
        self.a = a = V.vfl_layernorm_args() if kind == "norm" else V.vfl_residual_args()
        a.dtype, a.rows, a.cols, a.eps = (V.VFL_F32, V.VFL_BF16)[dt == "bf16"], rows, cols, EPS
        new = lambda values=None, extra=0: Mat(dt, rows, cols, (ld or cols) + extra, lead, values)  # noqa: E731
        self.x = new(activations(rng, rows, cols))
        self.y, self.dx = new(extra=1), new()
        self.dy = new(rng.normal(size=(rows, cols)) * 1e-2, 2)
        self.m = {"x": self.x, "y": self.y, "dy": self.dy, "dx": self.dx}
        if kind == "residual":
            self.r, self.s, self.dr = new(activations(rng, rows, cols)), new(), new(extra=3)
            self.ds = new(rng.normal(size=(rows, cols)) * 1e-2)
            self.m.update(r=self.r, s=self.s, dr=self.dr, ds=self.ds)
            key(a.drop, p)
        self.gamma = f32(cols, (1 + 0.1 * rng.normal(size=cols)).astype(np.float32))
        self.beta = f32(cols, (0.1 * rng.normal(size=cols)).astype(np.float32))
        self.g64 = stored(self.gamma, cols) if affine else np.ones(cols)
        self.b64 = stored(self.beta, cols) if affine else np.zeros(cols)
        if affine:
            a.gamma, a.beta = self.gamma.data_ptr(), self.beta.data_ptr()
        self.stats, self.dgamma, self.dbeta = f32(2 * rows), f32(cols), f32(cols)
        a.stats, a.dgamma, a.dbeta = (t.data_ptr() for t in (self.stats, self.dgamma, self.dbeta))
        n = V.vfl_norm_workspace_size(rows, cols)
        # 0xff bytes: NaN wherever a partial sum is read that was not written
        self.ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = self.ws.data_ptr(), n
        self.nws = n
        for name, m in self.m.items():
            m.put(getattr(a, name))

    def forward(self, stream=0):
        (self.V.vfl_layernorm_forward if self.kind == "norm" else self.V.vfl_residual_forward)(self.a, stream)

    def backward(self, stream=0):
        (self.V.vfl_layernorm_backward if self.kind == "norm" else self.V.vfl_residual_backward)(self.a, stream)

    def st(self):
        return stored(self.stats, 2 * self.rows).reshape(self.rows, 2)

    def guards(self):
        for m in self.m.values():
            m.assert_guard()
        assert bool((self.ws[self.nws:] == 0xFF).all())

    def check_forward(self, x=None, r=None):
        x = self.x.np() if x is None else x
        if self.kind == "norm":
            v, ev = x, np.zeros_like(x)
        else:
            r = self.r.np() if r is None else r
            k = keep(self.p, self.rows, self.cols)
            xd = R.dropout(x, self.p, k)
            v = r + xd
            ev = 2 * U * np.abs(xd) * (self.p > 0) + U * np.abs(v)
            if self.a.s.data:
                close(self.s.np(), v, SLACK * ev, "s", self.dt)
        y, stats = R.layer_norm(v, self.g64, self.b64, EPS)
        e_y, e_st = norm_bounds(v, ev, self.g64, self.b64)
        close(self.y.np(), y, e_y, "y", self.dt)
        if self.a.stats:
            close(self.st(), stats, e_st, "stats")

    def check_backward(self, v=None, dy=None, ds=None):
        v = (self.x if self.kind == "norm" else self.s).np() if v is None else v
        dy = self.dy.np() if dy is None else dy
        st = self.st()
        e_dx, e_dg, e_db = grad_bounds(v, st, self.g64, dy)
        dx, dg, db = R.layer_norm_backward(v, st, self.g64, dy)
        if self.kind == "norm":
            if self.a.dx.data:
                close(self.dx.np(), dx, e_dx, "dx", self.dt)
        else:
            ds = (self.ds.np() if self.a.ds.data else 0.0) if ds is None else ds
            dr = dx + ds
            e_dr = e_dx + SLACK * U * np.abs(dr)
            if self.a.dr.data:
                close(self.dr.np(), dr, e_dr, "dr", self.dt)
            if self.a.dx.data:
                k = keep(self.p, self.rows, self.cols)
                want = R.dropout(dr, self.p, k)
                got = self.dx.np()
                assert (got[~k] == 0).all()
                e = R.dropout(e_dr, self.p, k) + 2 * U * np.abs(want) * (self.p > 0)
                close(got, want, e, "dx", self.dt)
        if self.a.dgamma:
            close(stored(self.dgamma, self.cols), dg, e_dg, "dgamma")
        if self.a.dbeta:
            close(stored(self.dbeta, self.cols), db, e_db, "dbeta")


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("rows,cols,ld,lead", SHAPES)
def test_layer_norm(V, dt, rows, cols, ld, lead):
    c = Call(V, "norm", dt, rows, cols, ld, lead)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    c.guards()


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("rows,cols,ld,lead", SHAPES)
def test_residual(V, dt, p, rows, cols, ld, lead):
    c = Call(V, "residual", dt, rows, cols, ld, lead, p)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    c.guards()


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("rows,cols", [(40_000, 24), (20_000, 136), (6000, 520), (2600, 1500)])
def test_many_rows(V, dt, rows, cols):
    """More rows than one round of workgroups takes; the weights' gradients
    bitwise the same from run to run."""
    c = Call(V, "residual", dt, rows, cols, p=0.2)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    first = [t.clone() for t in (c.dgamma, c.dbeta, c.dx.t, c.dr.t)]
    c.ws.fill_(0xFF)
    c.backward()
    assert all(torch.equal(a, b) for a, b in zip(first, (c.dgamma, c.dbeta, c.dx.t, c.dr.t)))


@pytest.mark.parametrize("dt", DTS)
def test_no_rows(V, dt):
    c = Call(V, "residual", dt, 0, 40)
    c.forward()
    c.backward()
    assert (stored(c.dgamma, 40) == 0).all() and (stored(c.dbeta, 40) == 0).all()


OPTIONAL = [("norm", ["stats"], []), ("norm", [], ["dx"]), ("norm", [], ["dgamma"]), ("norm", [], ["dbeta"]),
            ("norm", [], ["dgamma", "dbeta"]), ("residual", ["s"], ["ds"]), ("residual", ["s", "stats"], ["dx"]),
            ("residual", [], ["dr"]), ("residual", [], ["dr", "dx"]), ("residual", [], ["dgamma", "dbeta"]),
            ("residual", [], ["ds", "dgamma"])]


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("cols", [50, 640])
@pytest.mark.parametrize("kind,no_fwd,no_bwd", OPTIONAL)
def test_optional_operands(V, dt, cols, kind, no_fwd, no_bwd):
    """Absent operands are neither read nor written, the others do not change."""
    def clear(c, names):
        for n in names:
            f = getattr(c.a, n)
            if isinstance(f, V.vfl_matrix):
                f.data = None
            else:
                setattr(c.a, n, None)

    c = Call(V, kind, dt, 70, cols, p=0.25)
    clear(c, no_fwd)
    c.forward()
    c.check_forward()
    for n in no_fwd:
        buf = getattr(c, n)
        assert bool(((buf.t if isinstance(buf, Mat) else buf) == Mat.GUARD).all())
    c = Call(V, kind, dt, 70, cols, p=0.25)
    c.forward()
    clear(c, no_bwd)
    c.backward()
    c.check_backward()
    for n in set(no_bwd) - {"ds"}:
        buf = getattr(c, n)
        assert bool(((buf.t if isinstance(buf, Mat) else buf) == Mat.GUARD).all())


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("cols", [24, 1032])
def test_without_weights(V, dt, cols):
    c = Call(V, "residual", dt, 50, cols, p=0.1, affine=False)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("cols", [5, 100, 1000, 5000])
def test_in_place(V, dt, cols):
    """Outputs over inputs: s over r, y over x; dr over ds, dx over dy; a layer
    norm's y over x and dx over dy."""
    ref = Call(V, "residual", dt, 90, cols, p=0.3)
    ref.forward()
    ref.backward()
    c = Call(V, "residual", dt, 90, cols, p=0.3)
    c.r.put(c.a.s)
    c.x.put(c.a.y)
    c.forward()
    assert torch.equal(c.r.t, ref.s.t) and torch.equal(c.x.t, ref.y.t)
    c.ds.put(c.a.dr)
    c.dy.put(c.a.dx)
    c.backward()
    assert torch.equal(c.ds.t, ref.dr.t) and torch.equal(c.dy.t, ref.dx.t)
    assert torch.equal(c.dgamma, ref.dgamma) and torch.equal(c.dbeta, ref.dbeta)
    ref = Call(V, "norm", dt, 90, cols)
    ref.forward()
    ref.backward()
    c = Call(V, "norm", dt, 90, cols)
    c.dy.put(c.a.dx)
    c.forward()
    c.backward()
    assert torch.equal(c.dy.t, ref.dx.t) and torch.equal(c.dgamma, ref.dgamma)
    c.x.put(c.a.y)
    c.forward()
    assert torch.equal(c.x.t, ref.y.t)


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("cols", [40, 3000])
def test_infinities_and_nan_stay_in_their_rows(V, dt, cols):
    """A row with an infinity or a NaN gives NaN there and nowhere else."""
    c = Call(V, "norm", dt, 20, cols)
    clean = Call(V, "norm", dt, 20, cols)
    clean.forward()
    c.x.t[3, 1] = float("inf")
    c.x.t[8, cols - 1] = float("nan")
    c.forward()
    rest = [i for i in range(20) if i not in (3, 8)]
    assert torch.equal(c.y.t[rest], clean.y.t[rest])
    assert bool(c.y.t[3].isnan().all()) and bool(c.y.t[8].isnan().all())
    c.backward()
    clean.backward()
    assert torch.equal(c.dx.t[rest], clean.dx.t[rest])


@pytest.mark.parametrize("dt", DTS)
def test_dropped_branch_does_not_leak_into_the_sum(V, dt):
    """Infinities and NaN at dropped places of the branch leave s, y untouched."""
    c = Call(V, "residual", dt, 30, 300, p=0.5)
    k = keep(0.5, 30, 300)
    vals = c.x.np()
    vals[~k] = np.where(np.arange((~k).sum()) % 2, np.nan, -np.inf)
    c.x.t.copy_(torch.from_numpy(vals))
    c.forward()
    c.check_forward(x=np.where(k, vals, 0.0))


@pytest.mark.parametrize("dt", DTS)
def test_everything_dropped(V, dt):
    """p = 1: the join passes r on; no gradient reaches the branch."""
    c = Call(V, "residual", dt, 30, 90, p=1.0)
    c.forward()
    assert torch.equal(c.s.t, c.r.t)
    c.check_forward()
    c.backward()
    assert bool((c.dx.t == 0).all())


@pytest.mark.parametrize("dt", DTS)
def test_large_mean_small_spread(V, dt):
    """Rows far from zero: the variance is taken around the mean."""
    rng = np.random.default_rng(1)
    c = Call(V, "norm", dt, 40, 700)
    c.x.t.copy_(torch.from_numpy(200.0 + rng.normal(size=(40, 700))))
    c.forward()
    c.check_forward()


@pytest.mark.parametrize("kind", ["norm", "residual"])
@pytest.mark.parametrize("rows,cols", [(6, 37), (3, 1100)])
def test_gradients_against_differences(V, kind, rows, cols):
    """The float32 backward against central differences of the float64
    definition along random directions.  With step e = 1e-5 the truncation is
    below 1e-6 of the scale here (third derivatives over e^2) and the
    cancellation below 1e-9; the rest is the bound of the gradients themselves."""
    c = Call(V, kind, "f32", rows, cols, p=0.3)
    c.forward()
    c.backward()
    x, dy = c.x.np(), c.dy.np()
    k = keep(0.3, rows, cols)
    if kind == "residual":
        r, ds = c.r.np(), c.ds.np()

        def loss(x, r, g, b):
            s, y, _ = R.residual(x, r, 0.3, k, g, b, EPS)
            return (dy * y).sum() + (ds * s).sum()
        args, grads = [x, r, c.g64, c.b64], [c.dx.np(), c.dr.np()]
    else:
        def loss(x, g, b):
            return (dy * R.layer_norm(x, g, b, EPS)[0]).sum()
        args, grads = [x, c.g64, c.b64], [c.dx.np()]
    grads += [stored(c.dgamma, cols), stored(c.dbeta, cols)]
    rng = np.random.default_rng(9)
    for i, g in enumerate(grads):
        for _ in range(3):
            # a direction over the rows that have a variance
            d = rng.normal(size=args[i].shape)
            if d.ndim == 2 and rows > 4:
                d[rows // 2] = 0.0
            up, dn = ([a + s * 1e-5 * d if j == i else a for j, a in enumerate(args)] for s in (1, -1))
            want = (loss(*up) - loss(*dn)) / 2e-5
            scale = np.abs(g * d).sum()
            assert abs((g * d).sum() - want) <= (1e-6 + 400 * U) * scale + 1e-9


@pytest.mark.parametrize("dt", DTS)
def test_offsets_past_32_bits(V, dt):
    """Rows whose element offsets pass 2^32 (a slice of a very wide matrix)."""
    rows, cols, ld = 66_000, 24, 65_600
    c = Call(V, "norm", dt, rows, cols)
    big = torch.empty((rows, ld), dtype=DT[dt], device="cuda")
    first = ld - 40
    big[:, first:first + cols] = c.x.t
    c.forward()
    c.backward()
    y, dx, dg = c.y.t.clone(), c.dx.t.clone(), c.dgamma.clone()
    c.a.x.data, c.a.x.ld = big.data_ptr() + first * big.element_size(), ld
    c.a.y.data, c.a.y.ld = c.a.x.data, ld
    c.a.dx.data, c.a.dx.ld = c.a.x.data, ld
    c.backward()
    assert torch.equal(big[:, first:first + cols], dx) and torch.equal(c.dgamma, dg)
    big[:, first:first + cols] = c.x.t
    c.forward()
    assert torch.equal(big[:, first:first + cols], y)
    big[:, first:first + cols] = c.x.t
    d, small = V.vfl_dropout_args(), Mat(dt, rows, cols)
    d.dtype, d.rows, d.cols = c.a.dtype, rows, cols
    key(d.drop, 0.5)
    c.x.put(d.x)
    small.put(d.y)
    V.vfl_dropout(d)
    d.x.data, d.x.ld = c.a.x.data, ld
    d.y.data, d.y.ld = c.a.x.data, ld
    V.vfl_dropout(d)
    assert torch.equal(big[:, first:first + cols], small.t)


def test_calls_follow_their_stream(V):
    """Inputs written and outputs read on another stream than the default."""
    c = Call(V, "residual", "bf16", 5000, 256, p=0.1)
    x = c.x.t.clone()
    c.forward()
    c.backward()
    want = [t.clone() for t in (c.y.t, c.dx.t, c.dgamma)]
    c.x.t.zero_()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        for _ in range(20):                      # work that the calls have to wait for
            c.x.t.add_(1.0)
        c.x.t.copy_(x)
        c.forward(st.cuda_stream)
        c.backward(st.cuda_stream)
        got = [t.clone() for t in (c.y.t, c.dx.t, c.dgamma)]
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_backward_in_a_replayed_graph(V):
    c = Call(V, "residual", "bf16", 4000, 192, p=0.2)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s = torch.cuda.current_stream().cuda_stream
        c.forward(s)
        c.backward(s)
    outs = (c.y.t, c.dx.t, c.dr.t, c.dgamma[:192], c.dbeta[:192])
    for i in range(4):
        c.x.t.mul_(1.5)
        c.forward()
        c.backward()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


# widths at which a row takes another number of chunks a lane or of wavefronts,
# one chunk more, and one that ends inside a chunk; more rows than the backward
# pass reads twice
EDGES = [8, 9, 16, 17, 32, 64, 72, 128, 136, 256, 264, 511, 512, 520, 1024, 1032, 1535, 1536, 1544, 3071, 3080, 4096,
         4104, 8192, 8193, 9000, 16384, 16385]


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("cols", EDGES)
def test_widths_where_the_layout_changes(V, dt, cols):
    rows = 1540 if cols > 1024 else 1100
    c = Call(V, "residual", dt, rows, cols, p=0.2)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    c.guards()
    few = Call(V, "norm", dt, 5, cols, (cols + 7) // 8 * 8, 1)
    few.forward()
    few.check_forward()
    few.backward()
    few.check_backward()
    few.guards()


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("rows,cols", [(1100, 24), (1600, 1300), (1600, 9000), (40, 20000)])
def test_in_place_with_many_rows(V, dt, rows, cols):
    """dx over dy and dr over ds, whichever way the weights' gradients are made."""
    ref = Call(V, "residual", dt, rows, cols, p=0.3)
    ref.forward()
    ref.backward()
    c = Call(V, "residual", dt, rows, cols, p=0.3)
    c.forward()
    c.ds.put(c.a.dr)
    c.dy.put(c.a.dx)
    c.backward()
    assert torch.equal(c.ds.t, ref.dr.t) and torch.equal(c.dy.t, ref.dx.t)
    assert torch.equal(c.dgamma, ref.dgamma) and torch.equal(c.dbeta, ref.dbeta)


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("cols", [3, 13, 100, 1001, 9001])
def test_values_between_rows_have_no_influence(V, dt, cols):
    """NaN behind every row's end (read along with a row's last chunk)."""
    rows = 23
    ref = Call(V, "residual", dt, rows, cols, cols + 9, 0, p=0.3)
    ref.forward()
    ref.backward()
    c = Call(V, "residual", dt, rows, cols, cols + 9, 0, p=0.3)
    for m in (c.x, c.r, c.s, c.dy, c.ds):
        m.buf[:rows * m.ld].view(rows, m.ld)[:, cols:] = float("nan")
    c.forward()
    c.backward()
    for name in ("y", "s", "dr", "dx"):
        assert torch.equal(c.m[name].t, ref.m[name].t)
    assert torch.equal(c.stats, ref.stats) and torch.equal(c.dgamma, ref.dgamma) and torch.equal(c.dbeta, ref.dbeta)
    d, y = V.vfl_dropout_args(), Mat(dt, rows, cols)
    d.dtype, d.rows, d.cols = c.a.dtype, rows, cols
    key(d.drop, 0.5)
    c.x.put(d.x)
    y.put(d.y)
    V.vfl_dropout(d)
    assert not bool(y.t.isnan().any())


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("rows,cols", [(1537, 1025), (1538, 1600), (1541, 2048), (1543, 1800), (2049, 2041), (1539, 2049),
                                       (1537, 8191)])
def test_rows_that_leave_part_of_a_workgroup_idle(V, dt, rows, cols):
    c = Call(V, "residual", dt, rows, cols, (cols + 15) // 8 * 8 + 1, 3, p=0.4)
    c.forward()
    c.backward()
    c.check_backward()
    c.guards()
    dgamma, dbeta = c.dgamma.clone(), c.dbeta.clone()
    c.backward()
    assert torch.equal(dgamma, c.dgamma) and torch.equal(dbeta, c.dbeta)       # the same sums in the same order
    c.a.dr.data = c.a.dx.data = None                                           # weights' gradients alone
    c.dgamma.fill_(0.0)
    c.dbeta.fill_(0.0)
    c.backward()
    assert torch.equal(dgamma[:cols], c.dgamma[:cols]) and torch.equal(dbeta[:cols], c.dbeta[:cols])


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("cols", [1, 5, 8, 9, 16, 24, 64, 72, 128, 129, 256, 260, 500, 512, 1000])
@pytest.mark.parametrize("rows", [770, 1281, 1999])
def test_narrow_rows_by_either_way_of_the_weights_gradients(V, dt, rows, cols):
    c = Call(V, "norm", dt, rows, cols, (cols + 7) // 8 * 8, 1)
    c.forward()
    c.backward()
    c.check_backward()
    c.guards()


@pytest.mark.parametrize("rows,cols", [(5, 40), (2100, 40)])
def test_an_earlier_error_of_the_caller_is_not_this_calls(V, rows, cols):
    """A failure that the caller has not asked for yet is neither reported by a
    call that succeeds nor taken from the caller."""
    lib = V.library()
    c = Call(V, "residual", "f32", rows, cols, p=0.2)
    n = Call(V, "norm", "f32", rows, cols)
    y = Mat("f32", rows, cols)
    d = V.vfl_dropout_args()
    d.dtype, d.rows, d.cols = V.VFL_F32, rows, cols
    key(d.drop, 0.5)
    c.x.put(d.x)
    y.put(d.y)
    torch.cuda.synchronize()
    try:
        assert lib.hipSetDevice(-1) != 0             # refused on the host
        before = lib.hipPeekAtLastError()
        assert before != 0
        for call in (lambda: V.vfl_dropout(d), c.forward, c.backward, n.forward, n.backward):
            call()
            assert lib.hipPeekAtLastError() == before
    finally:
        lib.hipGetLastError()
    torch.cuda.synchronize()
    assert ((y.np() != 0) == (keep(0.5, rows, cols) & (c.x.np() != 0))).all()
    for m in (c, n):
        m.check_forward()
        m.check_backward()


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("rows", [9, 2100])
@pytest.mark.parametrize("cols", [1, 4, 8, 13, 100, 1001, 1500])
def test_backward_of_huge_constant_rows(V, dt, rows, cols):
    """Rows without variance far from zero: (x - mean) * k is 0 at every column,
    and what lies past a row's end must not enter its sums as mean * k, which is
    infinite in float32."""
    c = Call(V, "residual", dt, rows, cols, p=0.2)
    c.forward()
    c.s.t[[0, rows // 2, rows - 1]] = 2.0 ** 121
    stats = R.layer_norm(c.s.np(), 1.0, 0.0, EPS)[1]
    c.stats[:2 * rows] = torch.from_numpy(stats.reshape(-1)).float()
    c.backward()
    c.check_backward()
    assert bool(c.dr.t.isfinite().all()) and bool(c.dgamma[:cols].isfinite().all())


# ------------------------------------------------------------- large batches
class Large(Call):
    """Inputs made on the device; checked at sampled rows (results of a row
    depend on that row alone) and, for the weights' gradients, in float64 on the
    device."""

    def __init__(self, V, kind, dt, rows, cols, ld=0, p=0.0):
        self.V, self.kind, self.dt, self.rows, self.cols, self.p = V, kind, dt, rows, cols, p
        g = torch.Generator(device="cuda").manual_seed(rows * 31 + cols)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.a = a = V.vfl_layernorm_args() if kind == "norm" else V.vfl_residual_args()
        a.dtype, a.rows, a.cols, a.eps = (V.VFL_F32, V.VFL_BF16)[dt == "bf16"], rows, cols, EPS

        def new(values=None):
            m = Mat(dt, rows, cols, ld)
            if values is not None:
                m.t.copy_(values)
            return m

        act = lambda: rnd(rows, cols) * torch.exp(0.5 * rnd(cols)) + 0.5 * rnd(rows, 1)  # noqa: E731
        self.x, self.y, self.dx, self.dy = new(act()), new(), new(), new(rnd(rows, cols) * 1e-2)
        self.m = {"x": self.x, "y": self.y, "dy": self.dy, "dx": self.dx}
        if kind == "residual":
            self.r, self.s, self.dr, self.ds = new(act()), new(), new(), new(rnd(rows, cols) * 1e-2)
            self.m.update(r=self.r, s=self.s, dr=self.dr, ds=self.ds)
            key(a.drop, p)
        self.gamma, self.beta = f32(cols), f32(cols)
        self.gamma[:cols], self.beta[:cols] = 1 + 0.1 * rnd(cols), 0.1 * rnd(cols)
        self.g64, self.b64 = stored(self.gamma, cols), stored(self.beta, cols)
        a.gamma, a.beta = self.gamma.data_ptr(), self.beta.data_ptr()
        self.stats, self.dgamma, self.dbeta = f32(2 * rows), f32(cols), f32(cols)
        a.stats, a.dgamma, a.dbeta = (t.data_ptr() for t in (self.stats, self.dgamma, self.dbeta))
        self.nws = V.vfl_norm_workspace_size(rows, cols)
        self.ws = torch.full((self.nws + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = self.ws.data_ptr(), self.nws
        for name, m in self.m.items():
            m.put(getattr(a, name))
        # the first and the last rows, and some between
        n = min(rows, 40)
        between = np.random.default_rng(rows).integers(0, rows, 60)
        self.sel = np.unique(np.concatenate([np.arange(n), between, np.arange(rows - n, rows)]))

    def at(self, m):
        return m.t[torch.from_numpy(self.sel).cuda()].double().cpu().numpy()

    def keep(self):
        return R.keep_mask(self.p, KEY["seed"], KEY["step"], KEY["tag"], KEY["row0"] + self.sel, self.cols)

    def check_forward(self):
        v = self.at(self.x)
        ev = np.zeros_like(v)
        if self.kind == "residual":
            xd = R.dropout(v, self.p, self.keep())
            v = self.at(self.r) + xd
            ev = 2 * U * np.abs(xd) * (self.p > 0) + U * np.abs(v)
            close(self.at(self.s), v, SLACK * ev, "s", self.dt)
        y, stats = R.layer_norm(v, self.g64, self.b64, EPS)
        e_y, e_st = norm_bounds(v, ev, self.g64, self.b64)
        close(self.at(self.y), y, e_y, "y", self.dt)
        close(self.st()[self.sel], stats, e_st, "stats")

    def check_backward(self):
        v = self.x if self.kind == "norm" else self.s
        vs, dy, st = self.at(v), self.at(self.dy), self.st()[self.sel]
        e, _, _ = grad_bounds(vs, st, self.g64, dy)
        d, _, _ = R.layer_norm_backward(vs, st, self.g64, dy)
        if self.kind == "residual":
            if self.a.ds.data:
                d = d + self.at(self.ds)
            e = e + SLACK * U * np.abs(d)
            if self.a.dr.data:
                close(self.at(self.dr), d, e, "dr", self.dt)
            k = self.keep()
            d, e = R.dropout(d, self.p, k), R.dropout(e, self.p, k)
            e = e + 2 * U * np.abs(d) * (self.p > 0)
        if self.a.dx.data:
            close(self.at(self.dx), d, e, "dx", self.dt)
        # as in grad_bounds, over all rows
        st = self.stats[:2 * self.rows].double().view(-1, 2)
        dy = self.dy.t.double()
        t = (v.t.double() - st[:, :1]) * st[:, 1:] * dy
        chain = min(self.rows, 512) + 32
        for name, terms, roundings in (("dgamma", t, chain + 4), ("dbeta", dy, chain)):
            if getattr(self.a, name):
                want, bound = terms.sum(0), SLACK * roundings * U * terms.abs().sum(0) + 1e-37
                close(stored(getattr(self, name), self.cols), want.cpu().numpy(), bound.cpu().numpy(), name)


# more rows than a round of forward workgroups takes, so that they go on to a next
# row (1 to 64 lanes a row, one and two chunks a lane, several wavefronts a row),
# with whole and partial last chunks; results too large to leave the L2s early
LARGE = [(1_050_001, 5), (1_050_001, 8), (530_001, 13), (270_001, 30), (140_001, 64), (70_001, 100), (70_001, 128),
         (35_001, 200), (44_001, 200), (33_001, 256), (17_001, 500), (17_001, 512), (8_501, 1000), (9_001, 1024),
         (66_001, 520), (33_001, 1032), (4_201, 2048), (3_001, 1536), (14_001, 4104), (9_001, 4096), (3_001, 5001),
         (1_501, 8192)]


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("kind", ["norm", "residual"])
@pytest.mark.parametrize("rows,cols", LARGE)
def test_large_batches(V, kind, dt, rows, cols):
    c = Large(V, kind, dt, rows, cols, p=0.3 if kind == "residual" else 0.0)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    c.guards()


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("rows,cols", [(210_001, 167), (70_001, 512), (4_300_001, 7)])
def test_dropout_of_more_chunks_than_threads(V, dt, rows, cols):
    """Threads step on to further (row, chunk) pairs."""
    p = 0.25
    x = Mat(dt, rows, cols)
    x.t.copy_(torch.rand((rows, cols), generator=torch.Generator(device="cuda").manual_seed(cols), device="cuda") + 0.5)
    y = Mat(dt, rows, cols)
    a = V.vfl_dropout_args()
    a.dtype, a.rows, a.cols = (V.VFL_F32, V.VFL_BF16)[dt == "bf16"], rows, cols
    key(a.drop, p)
    x.put(a.x)
    y.put(a.y)
    V.vfl_dropout(a)
    # everywhere: 0, or the element times the scale, rounded once to float32 and
    # once to the type
    want = (x.t.float() * float(np.float32(R.scale(p)))).to(DT[dt])
    kept = y.t != 0
    assert torch.equal(y.t, torch.where(kept, want, torch.zeros_like(want)))
    assert abs(kept.float().mean().item() - (1 - p)) < 0.002      # 30 million numbers: a deviation is 1e-4
    sel = np.unique(np.concatenate([np.arange(60), np.arange(rows - 60, rows), np.arange(0, rows, rows // 300)]))
    mask = R.keep_mask(p, KEY["seed"], KEY["step"], KEY["tag"], KEY["row0"] + sel, cols)
    assert (kept[torch.from_numpy(sel).cuda()].cpu().numpy() == mask).all()
    y.assert_guard()


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("rows,cols", [(2100, 50), (1300, 640), (1300, 1500), (800, 5001), (4300, 1000)])
@pytest.mark.parametrize("kind", ["norm", "residual"])
def test_optional_operands_of_many_rows(V, kind, dt, rows, cols):
    """Absent operands where partial weight gradients are summed in a second
    launch: neither read nor written, the others as the formulas say."""
    for names in {"norm": ["dx", "dgamma", "dbeta", "dgamma dbeta"],
                  "residual": ["ds", "dr", "dx", "dr dx", "ds dx", "ds dr", "dgamma", "dbeta", "ds dgamma", "dr dbeta",
                               "dgamma dbeta"]}[kind]:
        c = Large(V, kind, dt, rows, cols, cols + 3, p=0.25)
        c.forward()
        for n in names.split():
            f = getattr(c.a, n)
            if isinstance(f, V.vfl_matrix):
                f.data = None
            else:
                setattr(c.a, n, None)
        c.backward()
        c.check_backward()
        c.guards()
        for n in set(names.split()) - {"ds"}:
            buf = getattr(c, n)
            assert bool(((buf.t if isinstance(buf, Mat) else buf) == Mat.GUARD).all()), (names, n)


@pytest.mark.parametrize("rows,cols", [(60, 72), (2100, 72), (40, 1100)])
def test_residual_join_with_the_step_on_the_device_in_a_replayed_graph(V, rows, cols):
    """Both directions make the masks of step + *step_dev, at each replay anew."""
    p = 0.3
    c = Call(V, "residual", "f32", rows, cols, p=p)
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.a.drop.step_dev = step.data_ptr()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s = torch.cuda.current_stream().cuda_stream
        c.forward(s)
        c.backward(s)
        step.add_(1)
    xs = c.x.np()
    assert (xs != 0).mean() > 0.9
    for i in range(4):
        for t in (c.s.t, c.dx.t, c.y.t):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        k = keep(p, rows, cols, step=KEY["step"] + i)
        want = c.r.np() + R.dropout(xs, p, k)
        close(c.s.np(), want, SLACK * (2 * U * np.abs(R.dropout(xs, p, k)) + U * np.abs(want)), "s")
        dx, dr = c.dx.np(), c.dr.np()
        assert (dx[~k] == 0).all()
        close(dx, R.dropout(dr, p, k), 2.5 * U * np.abs(R.dropout(dr, p, k)), "dx")
        assert (dx[k & (dr != 0)] != 0).all()
