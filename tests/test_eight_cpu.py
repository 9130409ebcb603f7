"""Refusals of the operators of towers in 8 bits and of the softmax loss: every
invalid call returns before anything is launched, so these run without a GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def V():
    from paper_2510_12494_amd import vfl
    return vfl


BUF = (C.c_uint8 * 8192)()
BASE = (C.addressof(BUF) + 255) & ~255
CALLS = {"vfl_rmsnorm_forward": "vfl_rmsnorm_args", "vfl_rmsnorm_backward": "vfl_rmsnorm_args",
         "vfl_quantize": "vfl_quantize_args", "vfl_matmul8": "vfl_matmul8_args",
         "vfl_softmax_loss_forward": "vfl_softmax_loss_args", "vfl_softmax_loss_backward": "vfl_softmax_loss_args"}


def _args(V, call):
    a = getattr(V, CALLS[call])()
    a.dtype = V.VFL_F32
    for name, t in a._fields_:
        if t is V.vfl_matrix:
            getattr(a, name).data = BASE
        elif t is V.vfl_q8:
            getattr(a, name).data = getattr(a, name).scale = BASE
        elif t is C.c_void_p:
            setattr(a, name, BASE)
        elif name in ("rows", "m"):
            setattr(a, name, 4)
        elif name in ("cols", "dim", "n", "k", "classes"):
            setattr(a, name, 8)
    if hasattr(a, "eps"):
        a.eps = 1e-5
    if hasattr(a, "workspace_bytes"):
        a.workspace_bytes = 1 << 30
    return a


def _mats(cols, *names):
    out = []
    for m in names:
        out += [(m + ".data", BASE + 2, m + ":"), (m + ".ld", cols - 1, m + ":"), (m + ".ld", -1, m + ":"),
                (m + ".ld", 2**60, m + ":")]
    return out


def _eights(*names):
    out = []
    for m in names:
        out += [(m + ".data", BASE + 8, m + ":"), (m + ".ld", 64, m + ":"), (m + ".ld", 130, m + ":"),
                (m + ".ld", -128, m + ":"), (m + ".ld", 2**60, m + ":"), (m + ".scale", None, m + ":"),
                (m + ".scale", BASE + 4, m + ":"), (m + ".scale_ld", 8, m + ":"), (m + ".scale_ld", 24, m + ":"),
                (m + ".scale_ld", -16, m + ":")]
    return out


TYPE = [("dtype", 2, "dtype"), ("dtype", -1, "dtype")]
SIZE = TYPE + [("rows", -1, "rows"), ("rows", 2**41, "rows"), ("cols", 0, "cols"), ("cols", -3, "cols"),
               ("cols", 2**31 - 1, "cols")]
LOSS = TYPE + [("rows", -1, "rows"), ("rows", 2**21 + 1, "rows"), ("dim", 0, "cols"), ("dim", 32769, "cols"),
               ("classes", 0, "classes"), ("classes", 2**21 + 1, "classes"), ("bias", BASE + 2, "bias"),
               ("labels", BASE + 1, "labels"), ("labels", None, "labels"), ("loss", BASE + 2, "loss"),
               ("lse", BASE + 2, "lse"), ("workspace", BASE + 8, "workspace"), ("x.data", None, "x:"),
               ("w.data", None, "w:")] + _mats(8, "x", "w")
BAD = {
    "vfl_rmsnorm_forward": SIZE + [("cols", 32769, "cols"), ("gamma", BASE + 2, "gamma"), ("stats", BASE + 2, "stats"),
                                   ("eps", 0.0, "eps"), ("eps", float("nan"), "eps"), ("eps", float("inf"), "eps"),
                                   ("x.data", None, "x:")] + _mats(8, "x", "r", "s", "y") + _eights("q"),
    "vfl_rmsnorm_backward": SIZE + [("cols", 32769, "cols"), ("gamma", BASE + 2, "gamma"), ("dgamma", BASE + 1, "dgamma"),
                                    ("stats", None, "stats"), ("stats", BASE + 2, "stats"), ("s.data", None, "s:"),
                                    ("dy.data", None, "dy:"), ("workspace", BASE + 8, "workspace")]
    + _mats(8, "s", "dy", "ds", "dx"),
    "vfl_quantize": SIZE + [("x.data", None, "x:")] + _mats(8, "x") + _eights("q", "qt"),
    "vfl_matmul8": TYPE + [("m", -1, "rows"), ("m", 2**30 + 1, "m or n"), ("n", -1, "m or n"), ("n", 2**30 + 1, "m or n"),
                           ("k", 0, "k out"), ("k", 2**23 + 1, "k out"), ("bias", BASE + 1, "bias"),
                           ("workspace", BASE + 8, "workspace"), ("a.data", None, "a:"), ("b.data", None, "b:"),
                           ("c.data", None, "c:"), ("a.ld", 2**24, "a: ld"), ("b.ld", 2**24, "b: ld")]
    + _mats(8, "c") + _eights("a", "b"),
    "vfl_softmax_loss_forward": LOSS,
    "vfl_softmax_loss_backward": LOSS + [("lse", None, "lse"), ("dloss", BASE + 2, "dloss"), ("dbias", BASE + 2, "dbias")]
    + _mats(8, "dx", "dw"),
}


# an address differs from process to process: it takes no part in a test's name
@pytest.mark.parametrize("call,field,value,text", [(c, *bad) for c, bads in BAD.items() for bad in bads],
                         ids=lambda v: f"base+{v - BASE}" if isinstance(v, int) and BASE <= v < BASE + 64 else None)
def test_invalid_arguments_are_refused_with_their_reason(V, call, field, value, text):
    a = _args(V, call)
    at = a
    *path, last = field.split(".")
    for p in path:
        at = getattr(at, p)
    setattr(at, last, value)
    with pytest.raises(V.VflError) as e:
        getattr(V, call)(a)
    assert e.value.status == V.VFL_E_INVALID
    assert call in str(e.value) and text in str(e.value)
    assert text in V.vfl_last_error(None)


@pytest.mark.parametrize("call", sorted(CALLS))
def test_null_descriptor(V, call):
    assert getattr(V.library(), call)(None, None) == V.VFL_E_INVALID
    assert "args" in V.vfl_last_error(None)


def _without(a, V, *keep):
    for name, t in a._fields_:
        if name in ("s", "y", "q", "qt", "dx", "dw", "stats", "dgamma", "dbias", "loss", "lse") and name not in keep:
            if t is V.vfl_matrix or t is V.vfl_q8:
                getattr(a, name).data = None
            else:
                setattr(a, name, None)
    return a


@pytest.mark.parametrize("call,keep", [("vfl_rmsnorm_forward", ()), ("vfl_rmsnorm_backward", ("s", "stats")),
                                       ("vfl_quantize", ()), ("vfl_softmax_loss_forward", ()),
                                       ("vfl_softmax_loss_backward", ("lse",))])
def test_calls_without_an_output(V, call, keep):
    with pytest.raises(V.VflError) as e:
        getattr(V, call)(_without(_args(V, call), V, *keep))
    assert e.value.status == V.VFL_E_INVALID and "no output" in str(e.value)


def test_workspaces_that_are_too_small(V):
    a = _args(V, "vfl_rmsnorm_backward")
    a.rows = 100_000
    sizes = {"vfl_rmsnorm_backward": (a, V.vfl_norm_workspace_size(a.rows, a.cols))}
    a = _args(V, "vfl_matmul8")
    a.m, a.k = 100, 100_000                   # a sum that is cut into parts
    a.a.ld = a.b.ld = 0
    sizes["vfl_matmul8"] = (a, V.vfl_matmul8_workspace_size(a.m, a.n, a.k))
    for call in ("vfl_softmax_loss_forward", "vfl_softmax_loss_backward"):
        sizes[call] = (_args(V, call), V.vfl_softmax_loss_workspace_size(V.VFL_F32, 4, 8, 8))
    for call, (a, size) in sizes.items():
        assert size > 0
        a.workspace_bytes = size - 1
        for w in (BASE, None):
            a.workspace = w
            with pytest.raises(V.VflError) as e:
                getattr(V, call)(a)
            assert e.value.status == V.VFL_E_NOMEM and "workspace" in str(e.value)


@pytest.mark.parametrize("call", ["vfl_rmsnorm_forward", "vfl_quantize", "vfl_matmul8", "vfl_softmax_loss_forward"])
def test_no_rows_enqueue_nothing(V, call):
    a = _without(_args(V, call), V)
    for m in ("x", "r", "a", "c"):
        if hasattr(a, m):
            getattr(a, m).data = None
    setattr(a, "m" if call == "vfl_matmul8" else "rows", 0)
    getattr(V, call)(a)
    assert V.vfl_last_error(None) == ""


def test_no_rows_with_outputs_present(V):
    """A transpose of no rows has no blocks."""
    a = _args(V, "vfl_quantize")
    a.rows = 0
    V.vfl_quantize(a)
    assert V.vfl_last_error(None) == ""


def test_workspace_sizes_check_their_sizes(V):
    for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, 0), (2**31, 1, 1), (2**25, 2**25, 1), (2**30, 2**6 + 1, 1), (2**19, 2**18, 1),
                (1, 1, 2**24)):
        with pytest.raises(V.VflError):
            V.vfl_matmul8_workspace_size(*bad)
    for bad in ((2, 1, 1, 1), (0, -1, 1, 1), (0, 1, 0, 1), (0, 1, 1, 0), (0, 2**22, 1, 1), (0, 1, 1, 2**22), (0, 2**20, 1, 2**18)):
        with pytest.raises(V.VflError):
            V.vfl_softmax_loss_workspace_size(*bad)
    assert V.vfl_matmul8_workspace_size(0, 8, 8) == 0
    assert V.vfl_softmax_loss_workspace_size(0, 0, 8, 8) == 0


def test_workspaces_of_extreme_sizes(V):
    """The plans' own arithmetic at the limits, and sizes that grow with the problem."""
    w = V.vfl_softmax_loss_workspace_size
    for dt in (V.VFL_F32, V.VFL_BF16):
        for rows, dim, classes in ((1, 1, 1), (1, 1, 2**21), (2**21, 1, 1), (2**21, 32768, 2**16), (2**16, 32768, 2**21),
                                   (1, 32768, 2**21), (2**21, 32768, 1), (64, 250, 100_000), (8192, 256, 100_000)):
            size = w(dt, rows, dim, classes)
            # the operands' copies and a piece of G are in it, and no whole G of the large ones
            e = 4 if dt == V.VFL_F32 else 2
            assert size >= (rows + classes) * dim * e
            pairs = rows * max(classes // 64 + 2, 512) * 8                   # the forward's
            piece = max(1 << 30, rows * 512 * e + (1 << 20)) * 1.01 + 2**20
            sums = (64 * rows + 128 * 2**20 // max(dim, 1) + classes * 66) * (dim + 256) * 4
            assert size <= 2 * ((rows + classes) * (dim + 64) * e) + pairs + piece + sums + 2**30
    m = V.vfl_matmul8_workspace_size
    assert m(2**30, 2**6, 2**23) == m(1, 2**30, 2**23) == m(16, 2**30, 1) == 0
    assert 0 < m(128, 128, 2**23) <= 512 * 128 * 128 * 4
