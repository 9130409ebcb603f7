"""Cases that time the row operators of residual towers: dropout, layer norm
and the residual join of the two, with a plain form and a 64-bit reference.

    dropout         y = x * 65536 / (65536 - t) where kept, 0 elsewhere
    layer norm      h = (x - mean) * k, k = 1 / sqrt(var + eps); y = h * gamma + beta
    residual join   s = r + dropout(x), y = layer norm(s)

and their backward passes.  t = floor(65536 p + 1/2); element (row, col) is
kept when its 16-bit number is at least t.  The numbers of columns 8q .. 8q+7
are the eight halves (low half first) of one Philox4x32-10 block with key =
seed and counter = (step, row mod 2^32, q, 2^31 + (row >> 32) * 2^16 + tag), so
a mask follows from the sample's global row id and is never stored.

Fields of a case: `op` ("dropout", "norm", "norm_grad", "residual",
"residual_grad"), `dtype` of the activations (weights, statistics and the
weights' gradients are float32), `rows`, `cols`, `ld` (elements from row to
row: more than `cols` where rows are padded or a slice of a wider matrix),
`p`, and `train` (a forward pass that keeps the statistics for its backward).
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
STEP, TAG, ROW0 = 37, 2, 1_000_000
NAMES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, op, dtype, rows, cols, ld=0, p=0.0, train=True):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "cols": cols, "ld": ld or cols, "p": p,
            "train": train}


def listed():
    return [
        # the hidden layer of a first experiment on a small table (256-row
        # batches, float32): nothing but the latency of a call
        _case("dropout_tiny", "dropout", "f32", 256, 32, p=0.1),
        # a ragged last batch with a width of no round number
        _case("dropout_odd", "dropout", "f32", 4099, 333, p=0.25),
        # the widest hidden layer of unequal parties, four replicas of 8192 rows
        _case("dropout_wide", "dropout", "bf16", 32768, 1024, p=0.1),
        # scoring one sample
        _case("norm_one_row", "norm", "bf16", 1, 1024, train=False),
        # that tower's second layer in training
        _case("norm_hidden", "norm", "bf16", 32768, 512),
        # weight gradients of the smallest cut layer: latency again
        _case("norm_grad_tiny", "norm_grad", "f32", 256, 16),
        # a narrow cut layer over a large batch: many short rows
        _case("norm_grad_narrow", "norm_grad", "bf16", 262144, 64),
        # a 500-wide input layer in float32, rows padded to 16 bytes, ragged batch
        _case("norm_grad_padded", "norm_grad", "f32", 7813, 500, ld=504),
        # scoring a handful of samples through a residual block (no dropout)
        _case("residual_score", "residual", "bf16", 48, 1024, train=False),
        # a residual block of the widest layer in training
        _case("residual_hidden", "residual", "bf16", 32768, 1024, p=0.1),
        # few long rows of an odd width, float32
        _case("residual_grad_long", "residual_grad", "f32", 1537, 5001, p=0.5),
        # the backward pass of the widest block: the largest case
        _case("residual_grad_hidden", "residual_grad", "bf16", 32768, 1024, p=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges: operator, type, sizes and layout free."""
    while True:
        op = rng.choice(["dropout", "norm", "norm_grad", "residual", "residual_grad"])
        dtype = rng.choice(["f32", "bf16"])
        cols = _log(rng, 8, 16384)
        if rng.random() < 0.5:
            cols = max(8, cols // 16 * 16)
        rows = _log(rng, 1, 262144)
        if cols == 3072 or rows * cols * (4 if dtype == "f32" else 2) > 2**26:
            continue
        # whole rows, rows padded to 16 bytes, or a slice of a wider matrix
        ld = rng.choice([cols, cols, -(-cols // 8) * 8, cols + rng.randint(1, 64)])
        p = rng.choice([0.05, 0.1, 0.25, 0.5])
        train = rng.random() < 0.8
        if op in ("norm", "norm_grad") or (op == "residual" and not train):
            p = 0.0
        c = _case("", op, dtype, rows, cols, ld, p, train or op not in ("norm", "residual"))
        del c["name"]
        return c


# -------------------------------------------------------------------- inputs
def _matrix(case, values=None):
    """A [rows x cols] matrix of the case's layout."""
    m = torch.empty((case["rows"], case["ld"]), dtype=NAMES[case["dtype"]], device="cuda")
    m = m[:, :case["cols"]]
    if values is not None:
        m.copy_(values)
    return m


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols = case["rows"], case["cols"]
    rnd = lambda *size: torch.randn(size, generator=g, device="cuda")  # noqa: E731

    def activations():
        # per-column scales with a few large ones, a mean per row; the last
        # row of a larger batch is padding (constant: no variance)
        a = rnd(rows, cols) * torch.exp(0.5 * rnd(cols)) + 0.5 * rnd(rows, 1)
        if rows > 8:
            a[-1] = 0.0
        return _matrix(case, a)

    gradients = lambda: _matrix(case, rnd(rows, cols) * 1e-2)  # noqa: E731
    op = case["op"]
    st = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 0x5EED) % 2**64}
    if op != "residual_grad":
        st["x"] = activations()
    if op == "residual":
        st["r"] = activations()
    if op != "dropout":
        st["gamma"] = 1.0 + 0.1 * rnd(cols)
        st["beta"] = 0.1 * rnd(cols)
    if op in ("norm_grad", "residual_grad"):
        if op == "residual_grad":
            st["s"] = activations()
            st["ds"] = gradients()
        st["dy"] = gradients()
        # what the forward pass left: mean and k = 1 / sqrt(var + eps) per row
        v = st["x" if op == "norm_grad" else "s"].double()
        st["stats"] = torch.stack([v.mean(1), (v.var(1, unbiased=False) + EPS).rsqrt()], 1).float()
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _describe(st)
    return st


def _describe(st):
    """Output buffers, the workspace of the weights' gradients and the call's
    descriptor: what a program sets up once per layer."""
    from paper_2510_12494_amd import vfl as V
    c = st["case"]
    op, rows, cols = c["op"], c["rows"], c["cols"]
    f32 = dict(dtype=torch.float32, device="cuda")
    st["V"] = V
    if op == "dropout":
        a = V.vfl_dropout_args()
        out = {"y": _matrix(c)}
    elif op == "norm":
        a = V.vfl_layernorm_args()
        out = {"y": _matrix(c)}
    elif op == "norm_grad":
        a = V.vfl_layernorm_args()
        out = {"dx": _matrix(c)}
    elif op == "residual":
        a = V.vfl_residual_args()
        out = {"s": _matrix(c), "y": _matrix(c)}
    else:
        a = V.vfl_residual_args()
        out = {"dr": _matrix(c), "dx": _matrix(c)}
    if op in ("norm", "residual") and c["train"]:
        out["stats"] = torch.empty((rows, 2), **f32)
    if op in ("norm_grad", "residual_grad"):
        out["dgamma"], out["dbeta"] = torch.empty(cols, **f32), torch.empty(cols, **f32)
        size = V.vfl_norm_workspace_size(rows, cols)
        st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = st["workspace"].data_ptr(), size
    a.dtype = V.VFL_BF16 if c["dtype"] == "bf16" else V.VFL_F32
    a.rows, a.cols = rows, cols
    if op != "dropout":
        a.eps = EPS
        a.gamma, a.beta = st["gamma"].data_ptr(), st["beta"].data_ptr()
    if op in ("dropout", "residual", "residual_grad"):
        a.drop.p, a.drop.seed, a.drop.step, a.drop.tag, a.drop.row0 = c["p"], st["seed"], STEP, TAG, ROW0
    for k in ("x", "r", "s", "dy", "ds", "y", "dx", "dr"):
        t = out.get(k, st.get(k))
        if t is not None:
            m = getattr(a, k)
            m.data, m.ld = t.data_ptr(), t.stride(0)
    for k in ("stats", "dgamma", "dbeta"):
        t = out.get(k, st.get(k))
        if t is not None:
            setattr(a, k, t.data_ptr())
    st["args"], st["out"] = a, out
    st["call"] = {"dropout": V.vfl_dropout, "norm": V.vfl_layernorm_forward, "norm_grad": V.vfl_layernorm_backward,
                  "residual": V.vfl_residual_forward, "residual_grad": V.vfl_residual_backward}[op]


def run(state):
    if own:
        state["call"](state["args"], torch.cuda.current_stream().cuda_stream)
        return state["out"]
    return _plain(state)


# ---------------------------------------------------------------- plain form
M32 = 0xFFFFFFFF


def _mul32(c, m):
    """High and low words of the 64-bit products of 32-bit numbers, in int64."""
    a, b = (m >> 16) * c, (m & 0xFFFF) * c          # below 2^48
    lo = ((a & 0xFFFF) << 16) + b                   # below 2^49
    return (a >> 16) + (lo >> 32), lo & M32


def _factor(st):
    """What dropout multiplies each element with: 0 or 65536 / (65536 - t)."""
    c = st["case"]
    t = math.floor(c["p"] * 65536 + 0.5)
    row = torch.arange(ROW0, ROW0 + c["rows"], device="cuda")[:, None]
    q = torch.arange(-(-c["cols"] // 8), device="cuda")[None, :]
    w = [torch.full_like(row, STEP), row & M32, q, (1 << 31) + ((row >> 32) << 16) + TAG]
    k0, k1 = st["seed"] & M32, st["seed"] >> 32
    for _ in range(10):
        h0, l0 = _mul32(w[0], 0xD2511F53)
        h1, l1 = _mul32(w[2], 0xCD9E8D57)
        w = [h1 ^ w[1] ^ k0, l1, h0 ^ w[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    u = torch.stack([h for x in w for h in (x & 0xFFFF, x >> 16)], 2)
    keep = u.reshape(c["rows"], -1)[:, :c["cols"]] >= t
    return keep, 65536.0 / (65536 - t)


def _drop(st, v):
    if st["case"]["p"] == 0.0:
        return v
    keep, scale = _factor(st)
    return torch.where(keep, v * scale, 0.0)


def _norm(st, v):
    mean = v.mean(1, keepdim=True)
    d = v - mean
    k = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    return d * k * st["gamma"] + st["beta"], torch.cat([mean, k], 1)


def _norm_grad(st, v, dy):
    mean, k = st["stats"][:, :1], st["stats"][:, 1:]
    h = (v - mean) * k
    g = dy * st["gamma"]
    dv = k * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return dv, (dy * h).sum(0), dy.sum(0)


def _plain(st):
    c = st["case"]
    op, dt = c["op"], NAMES[c["dtype"]]
    f = {k: st[k].float() for k in ("x", "r", "s", "dy", "ds") if k in st}
    if op == "dropout":
        return {"y": _drop(st, f["x"]).to(dt)}
    if op in ("norm", "residual"):
        out, v = {}, f["x"]
        if op == "residual":
            v = f["r"] + _drop(st, v)
            out["s"] = v.to(dt)
        y, stats = _norm(st, v)
        out["y"] = y.to(dt)
        if c["train"]:
            out["stats"] = stats
        return out
    dv, dgamma, dbeta = _norm_grad(st, f["x" if op == "norm_grad" else "s"], f["dy"])
    if op == "norm_grad":
        return {"dx": dv.to(dt), "dgamma": dgamma, "dbeta": dbeta}
    dv = dv + f["ds"]
    return {"dr": dv.to(dt), "dx": _drop(st, dv).to(dt), "dgamma": dgamma, "dbeta": dbeta}


# ----------------------------------------------------------------- reference
def _kept(case, seed):
    """The kept elements, from 64-bit unsigned products on the host."""
    rows, cols = case["rows"], case["cols"]
    per = -(-cols // 8)
    t = int(np.floor(np.float64(case["p"]) * 65536.0 + 0.5))
    out = np.empty((rows, per * 8), dtype=bool)
    step = max(1, 65536 // per)
    mask, half = np.uint64(M32), np.uint64(32)
    for r0 in range(0, rows, step):
        n = min(step, rows - r0)
        row = np.repeat(np.arange(ROW0 + r0, ROW0 + r0 + n, dtype=np.uint64), per)
        c0 = np.full(n * per, STEP, dtype=np.uint64)
        c1 = row & mask
        c2 = np.tile(np.arange(per, dtype=np.uint64), n)
        c3 = np.uint64(0x80000000) | (row >> half) << np.uint64(16) | np.uint64(TAG)
        for i in range(10):
            ka = np.uint64(((seed & M32) + i * 0x9E3779B9) & M32)
            kb = np.uint64(((seed >> 32) + i * 0xBB67AE85) & M32)
            pa, pb = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
            c0, c1, c2, c3 = pb >> half ^ c1 ^ ka, pb & mask, pa >> half ^ c3 ^ kb, pa & mask
        words = np.stack([c0, c1, c2, c3], 1).astype("<u4")
        out[r0:r0 + n] = words.view("<u2").reshape(n, per * 8) >= t
    return torch.from_numpy(out[:, :cols]).cuda(), 65536.0 / (65536.0 - t)


def exact(case, seed):
    """The operators' definitions in float64."""
    st = _inputs(case, seed)
    op, n = case["op"], case["cols"]
    f = {k: v.double() for k, v in st.items() if torch.is_tensor(v)}
    keep, scale = _kept(case, st["seed"]) if case["p"] > 0 else (None, 1.0)
    drop = lambda v: v if keep is None else v.mul(scale).masked_fill_(~keep, 0.0)  # noqa: E731
    if op == "dropout":
        return {"y": drop(f["x"])}
    if op in ("norm", "residual"):
        v = f["x"] if op == "norm" else drop(f["x"]) + f["r"]
        mean = v.sum(1) / n
        k = (((v - mean[:, None]) ** 2).sum(1) / n + EPS) ** -0.5
        out = {"s": v} if op == "residual" else {}
        out["y"] = torch.addcmul(f["beta"], (v - mean[:, None]) * k[:, None], f["gamma"])
        if case["train"]:
            out["stats"] = torch.stack([mean, k], 1)
        return out
    mean, k = f["stats"].unbind(1)
    h = (f["x" if op == "norm_grad" else "s"] - mean[:, None]) * k[:, None]
    g = f["dy"] * f["gamma"]
    mg, mgh = g.sum(1) / n, (g * h).sum(1) / n
    dv = (g - mg[:, None] - h * mgh[:, None]) * k[:, None]
    weights = {"dgamma": (f["dy"] * h).sum(0), "dbeta": f["dy"].sum(0)}
    if op == "norm_grad":
        return {"dx": dv, **weights}
    dv = dv + f["ds"]
    return {"dr": dv, "dx": drop(dv.clone()), **weights}


# ---------------------------------------------------------------------- work
def work(case):
    """Bytes: each input and output once.  Operations per element: dropout 2;
    normalising 8 (mean 1, variance 3, the affine map 4); its backward 15 (h 2,
    g 1, the row's two sums 3, dx 5, the columns' two sums 4)."""
    rows, cols = case["rows"], case["cols"]
    el = rows * cols
    e = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    mats = {"dropout": 2, "norm": 2, "norm_grad": 3, "residual": 4, "residual_grad": 5}[op]
    flops = {"dropout": 2, "norm": 8, "norm_grad": 15, "residual": 9, "residual_grad": 16}[op]
    if op.startswith("residual") and case["p"] > 0:
        flops += 2
    nbytes = mats * el * e
    if op in ("norm", "residual"):
        nbytes += 8 * cols + (8 * rows if case["train"] else 0)
    elif op != "dropout":
        nbytes += 12 * cols + 8 * rows
    return {"bytes": nbytes, "flops": flops * el}
