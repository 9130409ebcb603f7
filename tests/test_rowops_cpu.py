"""Refusals of the row operators: every invalid call returns before anything
is launched, so these run without a GPU."""
import ctypes as C

import pytest

import numpy as np


@pytest.fixture(scope="module")
def V():
    from paper_2510_12494_amd import vfl
    return vfl


BUF = (C.c_uint8 * 4096)()
BASE = (C.addressof(BUF) + 255) & ~255


def _args(V, kind):
    a = {"dropout": V.vfl_dropout_args, "norm": V.vfl_layernorm_args, "residual": V.vfl_residual_args}[kind]()
    a.dtype, a.rows, a.cols = V.VFL_F32, 4, 8
    for name, t in a._fields_:
        if t is V.vfl_matrix:
            getattr(a, name).data = BASE
    if kind != "dropout":
        a.eps = 1e-5
        a.stats = a.dgamma = a.dbeta = a.workspace = BASE
        a.workspace_bytes = 1 << 20
    if kind != "norm":
        a.drop.p = 0.5
    return a


CALLS = {"vfl_dropout": "dropout", "vfl_layernorm_forward": "norm", "vfl_layernorm_backward": "norm",
         "vfl_residual_forward": "residual", "vfl_residual_backward": "residual"}
COMMON = [("dtype", 2, "dtype"), ("dtype", -1, "dtype"), ("rows", -1, "rows"), ("rows", 2**41, "rows"),
          ("cols", 0, "cols"), ("cols", -3, "cols"), ("cols", 2**31 - 1, "cols")]
DROP = [("drop.p", -0.1, "p must"), ("drop.p", 1.5, "p must"), ("drop.p", float("nan"), "p must"),
        ("drop.tag", 65536, "tag"), ("drop.row0", -1, "sample ids"), ("drop.row0", 2**47 - 3, "sample ids"),
        ("drop.step_dev", BASE + 2, "step_dev")]
NORM = [("gamma", BASE + 2, "gamma"), ("beta", BASE + 1, "beta"), ("stats", BASE + 4, "stats"),
        ("cols", 32769, "cols")]
FWD = [("eps", 0.0, "eps"), ("eps", -1e-5, "eps"), ("eps", float("nan"), "eps"), ("eps", float("inf"), "eps")]
BWD = [("stats", None, "stats"), ("dgamma", BASE + 2, "dgamma"), ("dbeta", BASE + 3, "dbeta"),
       ("workspace", BASE + 8, "workspace")]


def _mats(*names):
    out = []
    for m in names:
        out += [(m + ".data", BASE + 2, m + ":"), (m + ".ld", 7, m + ":"), (m + ".ld", -1, m + ":"),
                (m + ".ld", 2**60, m + ":")]
    return out


BAD = {"vfl_dropout": COMMON + DROP + _mats("x", "y") + [("x.data", None, "x:"), ("y.data", None, "y:")],
       "vfl_layernorm_forward": COMMON + NORM + FWD + _mats("x", "y") + [("x.data", None, "x:"), ("y.data", None, "y:")],
       "vfl_layernorm_backward": COMMON + NORM + BWD + _mats("x", "dy", "dx") + [("x.data", None, "x:"),
                                                                               ("dy.data", None, "dy:")],
       "vfl_residual_forward": COMMON + NORM + FWD + DROP + _mats("x", "r", "s", "y") + [
           ("x.data", None, "x:"), ("r.data", None, "r:"), ("y.data", None, "y:")],
       "vfl_residual_backward": COMMON + NORM + BWD + DROP + _mats("s", "dy", "ds", "dr", "dx") + [
           ("s.data", None, "s:"), ("dy.data", None, "dy:")]}


# an address differs from process to process: it takes no part in a test's name
@pytest.mark.parametrize("call,field,value,text", [(c, *bad) for c, bads in BAD.items() for bad in bads],
                         ids=lambda v: f"base+{v - BASE}" if isinstance(v, int) and BASE <= v < BASE + 64 else None)
def test_invalid_arguments_are_refused_with_their_reason(V, call, field, value, text):
    a = _args(V, CALLS[call])
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


@pytest.mark.parametrize("call,outs", [("vfl_layernorm_backward", ["dx"]), ("vfl_residual_backward", ["dr", "dx"])])
def test_backward_without_an_output_or_a_workspace(V, call, outs):
    a = _args(V, CALLS[call])
    a.rows = 100_000                          # a size that takes partial sums
    a.workspace_bytes = V.vfl_norm_workspace_size(a.rows, a.cols) - 1
    with pytest.raises(V.VflError) as e:
        getattr(V, call)(a)
    assert e.value.status == V.VFL_E_NOMEM and "workspace" in str(e.value)
    a.workspace = None
    with pytest.raises(V.VflError) as e:
        getattr(V, call)(a)
    assert e.value.status == V.VFL_E_NOMEM
    a.dgamma = a.dbeta = None
    for m in outs:
        getattr(a, m).data = None
    with pytest.raises(V.VflError) as e:
        getattr(V, call)(a)
    assert e.value.status == V.VFL_E_INVALID and "no output" in str(e.value)


def test_no_rows_enqueue_nothing(V):
    for call in ("vfl_dropout", "vfl_layernorm_forward", "vfl_residual_forward"):
        a = _args(V, CALLS[call])
        a.rows = 0
        for name, t in a._fields_:
            if t is V.vfl_matrix:
                getattr(a, name).data = None
        getattr(V, call)(a)
        assert V.vfl_last_error(None) == ""


def test_workspace_size(V):
    lib = V.library()
    assert lib.vfl_norm_workspace_size(4, 8, None) == V.VFL_E_INVALID
    for rows, cols in ((-1, 8), (4, 0), (4, V.VFL_NORM_MAX_COLS + 1), (2**41, 8)):
        with pytest.raises(V.VflError):
            V.vfl_norm_workspace_size(rows, cols)
    rng = np.random.default_rng(0)
    for _ in range(200):
        rows, cols = int(2 ** rng.uniform(0, 30)), int(2 ** rng.uniform(0, 15))
        n = V.vfl_norm_workspace_size(rows, cols)
        # whole pairs of float32 rows, and never a large share of the device
        assert n % (8 * cols) == 0 and n <= 512 << 20


def test_binding_matches_the_header_layout(V, tmp_path):
    """sizeof and offsetof of every descriptor, from a C program."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = [V.vfl_matrix, V.vfl_dropout_spec, V.vfl_dropout_args, V.vfl_layernorm_args, V.vfl_residual_args]
    lines = []
    for s in structs:
        lines.append(f'printf("%zu\\n", sizeof({s.__name__}));')
        lines += [f'printf("%zu\\n", offsetof({s.__name__}, {f[0]}));' for f in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "vfl.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", exe],
                   check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for s in structs:
        want.append(C.sizeof(s))
        want += [getattr(s, f[0]).offset for f in s._fields_]
    assert got == want


@pytest.mark.parametrize("cols", [1, 8, 64, 65, 500, 1024, 1025, 2400, 4096, 5001, 16384, 16392, 32768])
def test_a_workspace_serves_every_smaller_batch(V, cols):
    """Sizes never shrink with the rows."""
    last = 0
    for rows in list(range(0, 5000, 7)) + [2**k for k in range(13, 40)]:
        n = V.vfl_norm_workspace_size(rows, cols)
        assert n >= last
        last = n


def test_an_earlier_error_of_the_caller_is_not_this_calls(V):
    """A backward pass of no rows without weights launches nothing: it succeeds
    whatever the thread's last error is, and leaves that to the caller."""
    lib = V.library()
    assert lib.hipSetDevice(-1) != 0
    before = lib.hipPeekAtLastError()
    assert before != 0
    for call in ("vfl_layernorm_backward", "vfl_residual_backward"):
        a = _args(V, CALLS[call])
        a.rows, a.dgamma, a.dbeta = 0, None, None
        getattr(V, call)(a)
        assert V.vfl_last_error(None) == ""
        assert lib.hipPeekAtLastError() == before
    lib.hipGetLastError()
