"""Cases that time the operators of towers in 8 bits and of a head with many
classes: the root-mean-square norm with the residual's addition, matrices in 8
bits, their product, and the softmax cross-entropy of a linear head, with a
plain form and a 64-bit reference.

    rms norm        s = r + x, k = 1 / sqrt(mean(s^2) + eps), y = s * k * gamma, kept in
                    the storage type, in 8 bits, or both; and its backward pass
    quantize        a matrix in 8 bits, and the transpose in 8 bits
    matmul8         C = A B^T + bias, ReLU, of matrices in 8 bits
    softmax loss    z = x W^T + bias, loss = log(sum exp z) - z[label], and its
                    gradients with respect to x, W and bias

A matrix in 8 bits holds e4m3 values and one power of two for each block of 128
consecutive columns of a row: the smallest 2^e, e >= -127, that keeps the
block's magnitudes within 448.  Bytes are row-major, a row's length a multiple of
128 with zeros past its columns; the exponent of (row r, block b) is the byte
e + 127 at [b, r] of an array whose rows are a multiple of 16 long.

Fields of a case: `op` ("rms", "rms_grad", "quantize", "matmul8", "loss",
"loss_step": forward and backward), `dtype` ("f32", "bf16": of activations and
gradients, of the product's result, of the head's operands), the sizes (`rows`,
`cols`; `depth` of a product; `classes` of a head whose inputs have `cols`
columns), `ld` (elements from row to row), and what an operator keeps:
`train` (rms: s and the statistics, for the backward pass), `outs` (rms: "q",
"y" or "yq"; quantize: "q", "t" or "qt"), `bias` (a product's bias and ReLU).
"""
import math

import torch

own = False

EPS = 2.0 ** -17
BLOCK, TOP = 128, 448.0
NAMES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, op, dtype, rows, cols, **more):
    c = {"name": name, "op": op, "dtype": dtype, "rows": rows, "cols": cols, "ld": cols}
    c.update(more)
    return c


def listed():
    return [
        # scoring one sample: the input of a block's first product
        _case("rms_one_row", "rms", "bf16", 1, 1024, train=False, outs="q"),
        # a block of the widest layer in training, four replicas of 8192 rows
        _case("rms_hidden", "rms", "bf16", 32768, 1024, train=True, outs="q"),
        # its backward pass
        _case("rms_grad_hidden", "rms_grad", "bf16", 32768, 1024),
        # a 500-wide input layer in float32, rows padded to 16 bytes, ragged batch
        _case("quantize_odd", "quantize", "f32", 4099, 500, ld=504, outs="qt"),
        # the gradient of the widest layer, for the two products that read it
        _case("quantize_hidden", "quantize", "bf16", 32768, 1024, outs="qt"),
        # a layer of a block for one sample
        _case("matmul_one_row", "matmul8", "bf16", 1, 1024, depth=1024, bias=True),
        # a 1024 -> 512 layer of unequal parties, four replicas of 8192 rows
        _case("matmul_hidden", "matmul8", "bf16", 32768, 512, depth=1024, bias=True),
        # the weight gradient of the layer before it (500 inputs): few results, long sums
        _case("matmul_wgrad", "matmul8", "f32", 1024, 500, depth=32768, bias=False),
        # a wide tower: nothing but the matrix cores
        _case("matmul_wide", "matmul8", "bf16", 8192, 8192, depth=4096, bias=True),
        # scoring a handful of samples against a thousand classes, float32
        _case("loss_score", "loss", "f32", 48, 250, classes=1000),
        # a training step of odd sizes in float32
        _case("loss_step_odd", "loss_step", "f32", 1537, 333, classes=5003),
        # one batch against a table of 100k items: the largest case
        _case("loss_step_catalogue", "loss_step", "bf16", 8192, 256, classes=100_000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    n = _log(rng, lo, hi)
    return max(lo, n // 64 * 64) if rng.random() < 0.5 and n >= 64 else n


def draw(rng):
    """One more case of the listed ranges: operator, type, sizes and layout free."""
    while True:
        op = rng.choice(["rms", "rms_grad", "quantize", "matmul8", "matmul8", "loss", "loss_step", "loss_step"])
        dtype = rng.choice(["f32", "bf16"])
        e = 4 if dtype == "f32" else 2
        if op == "matmul8":
            rows, cols, depth = _size(rng, 1, 32768), _size(rng, 8, 8192), _size(rng, 8, 32768)
            if rows * cols * depth > 2**38 or max(rows, cols) * depth > 2**28 or rows * cols > 2**27:
                continue
            more = {"depth": depth, "bias": rng.random() < 0.6}
        elif op in ("loss", "loss_step"):
            rows, cols, classes = _size(rng, 1, 8192), _size(rng, 8, 1024), _size(rng, 2, 100_000)
            if rows * cols * classes > 2**37 or (dtype == "f32" and rows * cols * classes > 2**35):
                continue
            more = {"classes": classes}
        else:
            rows, cols = _size(rng, 1, 262144), _size(rng, 8, 16384)
            if rows * cols * e > 2**26:
                continue
            more = {}
            if op == "rms":
                more = {"train": rng.random() < 0.6, "outs": rng.choice(["q", "q", "y", "yq"])}
            elif op == "quantize":
                more = {"outs": rng.choice(["q", "t", "qt", "qt"])}
        # whole rows, rows padded to 16 bytes, or a slice of a wider matrix
        ld = rng.choice([cols, cols, -(-cols // 8) * 8, cols + rng.randint(1, 64)])
        c = _case("", op, dtype, rows, cols, **more)
        c["ld"] = ld
        del c["name"]
        return c


# -------------------------------------------------------------------- inputs
def _up(n, by):
    return -(-n // by) * by


def _matrix(dtype, rows, cols, ld=0, values=None):
    """A [rows x cols] matrix with ld elements from row to row."""
    m = torch.empty((rows, max(ld, cols)), dtype=NAMES[dtype], device="cuda")[:, :cols]
    if values is not None:
        m.copy_(values)
    return m


def _eight(v):
    """A float32 matrix in 8 bits: (e4m3 bytes, exponent bytes)."""
    rows, cols = v.shape
    wide = torch.zeros((rows, _up(cols, BLOCK)), device="cuda")
    wide[:, :cols] = v
    blocks = wide.view(rows, -1, BLOCK)
    # amax = m * 2^x, 1/2 <= m < 1: within 448 = 7/8 * 2^9 at e = x - 9, or one more
    m, x = torch.frexp(blocks.abs().amax(2))
    e = torch.where(m > 0, x - 9 + (m > TOP / 512), -127).clamp_(min=-127)
    q = torch.ldexp(blocks, -e[:, :, None]).to(torch.float8_e4m3fn)
    scale = torch.full((blocks.shape[1], _up(rows, 16)), 127, dtype=torch.uint8, device="cuda")
    scale[:, :rows] = (e + 127).T
    return q.view(rows, -1), scale


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dt, rows, cols, ld = case["op"], case["dtype"], case["rows"], case["cols"], case["ld"]
    rnd = lambda *size: torch.randn(size, generator=g, device="cuda")  # noqa: E731
    st = {"case": case}

    def activations(n=rows, k=cols):
        # per-column scales with a few large ones; the last row of a larger
        # batch is padding
        a = rnd(n, k) * torch.exp(0.5 * rnd(k))
        if n > 8:
            a[-1] = 0.0
        return a

    # rows that the model has learnt have small gradients
    gradients = lambda n=rows, k=cols: rnd(n, k) * torch.exp(1.5 * rnd(n, 1)) * 1e-3  # noqa: E731
    matrix = lambda v: _matrix(dt, rows, cols, ld, v)  # noqa: E731
    if op in ("rms", "rms_grad"):
        st["gamma"] = 1.0 + 0.1 * rnd(cols)
        if op == "rms":
            st["x"], st["r"] = matrix(activations()), matrix(activations())
        else:
            st["s"], st["dy"], st["ds"] = matrix(activations()), matrix(gradients()), matrix(gradients())
            st["stats"] = (st["s"].double().square().mean(1) + EPS).rsqrt().float()
    elif op == "quantize":
        st["x"] = matrix(gradients())
    elif op == "matmul8":
        # activations, or a weight's gradient: deltas and inputs, both transposed
        a, k = activations(rows, case["depth"]), case["depth"]
        b = rnd(cols, k) / math.sqrt(k) if case["bias"] else activations(cols, k)
        st["a"], st["b"] = _eight(a), _eight(b)
        if case["bias"]:
            st["bias"] = 0.1 * rnd(cols)
    else:
        n = case["classes"]
        w = rnd(n, cols) * (1.5 / math.sqrt(cols))
        # labels as a catalogue has them, a few far more frequent than most;
        # some samples already close to their class, some without a label, and
        # some classes withdrawn (no sample has them)
        u = torch.rand(rows, generator=g, device="cuda")
        label = (torch.exp(u * math.log(n + 1.0)) - 1).long().clamp_(0, n - 1)
        bias = 0.5 * rnd(n)
        gone = torch.rand(n, generator=g, device="cuda") < 0.02
        gone[label] = False
        bias[gone] = -math.inf
        near = 2.0 * torch.rand(rows, 1, generator=g, device="cuda")
        x = rnd(rows, cols) + near * w[label]
        label[torch.rand(rows, generator=g, device="cuda") < 0.03] = -1
        st["x"], st["w"] = matrix(x), _matrix(dt, n, cols, 0, w)
        st["bias"], st["label"] = bias, label.int()
        if op == "loss_step":
            # a mean over the batch, samples weighted
            st["dloss"] = (0.5 + torch.rand(rows, generator=g, device="cuda")) / rows
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _describe(st)
    return st


def _eight_out(rows, cols):
    return (torch.empty((rows, _up(cols, BLOCK)), dtype=torch.float8_e4m3fn, device="cuda"),
            torch.empty((_up(cols, BLOCK) // BLOCK, _up(rows, 16)), dtype=torch.uint8, device="cuda"))


def _describe(st):
    """Output buffers, workspaces and the calls' descriptors: what a program sets
    up once per layer."""
    from paper_2510_12494_amd import vfl as V
    c = st["case"]
    op, rows, cols = c["op"], c["rows"], c["cols"]
    f32 = dict(dtype=torch.float32, device="cuda")
    like = lambda n=rows, k=cols, ld=c["ld"]: _matrix(c["dtype"], n, k, ld)  # noqa: E731

    def put(m, t):
        m.data, m.ld = t.data_ptr(), t.stride(0)

    def put8(m, q):
        m.data, m.ld, m.scale, m.scale_ld = q[0].data_ptr(), q[0].stride(0), q[1].data_ptr(), q[1].stride(0)

    def workspace(size):
        st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = st["workspace"].data_ptr(), size

    out, kept = {}, {}
    if op in ("rms", "rms_grad"):
        a = V.vfl_rmsnorm_args()
        a.rows, a.cols, a.eps, a.gamma = rows, cols, EPS, st["gamma"].data_ptr()
        if op == "rms":
            put(a.x, st["x"])
            put(a.r, st["r"])
            if c["train"]:
                out["s"], out["stats"] = like(), torch.empty(rows, **f32)
                put(a.s, out["s"])
                a.stats = out["stats"].data_ptr()
            if "y" in c["outs"]:
                out["y"] = like()
                put(a.y, out["y"])
            if "q" in c["outs"]:
                kept["q"] = _eight_out(rows, cols)
                put8(a.q, kept["q"])
            calls = [V.vfl_rmsnorm_forward]
        else:
            out["dx"], out["dgamma"] = like(), torch.empty(cols, **f32)
            for k in ("s", "dy", "ds"):
                put(getattr(a, k), st[k])
            put(a.dx, out["dx"])
            a.stats, a.dgamma = st["stats"].data_ptr(), out["dgamma"].data_ptr()
            workspace(V.vfl_norm_workspace_size(rows, cols))
            calls = [V.vfl_rmsnorm_backward]
    elif op == "quantize":
        a = V.vfl_quantize_args()
        a.rows, a.cols = rows, cols
        put(a.x, st["x"])
        if "q" in c["outs"]:
            kept["q"] = _eight_out(rows, cols)
            put8(a.q, kept["q"])
        if "t" in c["outs"]:
            kept["t"] = _eight_out(cols, rows)
            put8(a.qt, kept["t"])
        calls = [V.vfl_quantize]
    elif op == "matmul8":
        a = V.vfl_matmul8_args()
        a.m, a.n, a.k = rows, cols, c["depth"]
        put8(a.a, st["a"])
        put8(a.b, st["b"])
        out["c"] = like()
        put(a.c, out["c"])
        if c["bias"]:
            a.bias, a.relu = st["bias"].data_ptr(), 1
        workspace(V.vfl_matmul8_workspace_size(rows, cols, c["depth"]))
        calls = [V.vfl_matmul8]
    else:
        a = V.vfl_softmax_loss_args()
        n = c["classes"]
        a.rows, a.dim, a.classes = rows, cols, n
        put(a.x, st["x"])
        put(a.w, st["w"])
        a.bias, a.labels = st["bias"].data_ptr(), st["label"].data_ptr()
        out["loss"], out["lse"] = torch.empty(rows, **f32), torch.empty(rows, **f32)
        a.loss, a.lse = out["loss"].data_ptr(), out["lse"].data_ptr()
        calls = [V.vfl_softmax_loss_forward]
        code = V.VFL_BF16 if c["dtype"] == "bf16" else V.VFL_F32
        if op == "loss_step":
            a.dloss = st["dloss"].data_ptr()
            out["dx"], out["dw"], out["dbias"] = like(), like(n, cols, cols), torch.empty(n, **f32)
            put(a.dx, out["dx"])
            put(a.dw, out["dw"])
            a.dbias = out["dbias"].data_ptr()
            calls.append(V.vfl_softmax_loss_backward)
        workspace(V.vfl_softmax_loss_workspace_size(code, rows, cols, n))
    a.dtype = V.VFL_BF16 if c["dtype"] == "bf16" else V.VFL_F32
    # the exponents of the rows that a matrix has
    for k, (q, scale) in kept.items():
        out[k], out[k + "_scale"] = q, scale[:, :q.shape[0]]
    st["args"], st["out"], st["calls"] = a, out, calls


def run(state):
    if own:
        stream = torch.cuda.current_stream().cuda_stream
        for call in state["calls"]:
            call(state["args"], stream)
        return state["out"]
    return _plain(state)


# ---------------------------------------------------------------- plain form
def _put_eight(out, key, v):
    out[key], scale = _eight(v)
    out[key + "_scale"] = scale[:, :v.shape[0]]


def _values(q):
    """What a matrix in 8 bits stands for, with the columns of its padding."""
    data, scale = q
    rows = data.shape[0]
    e = scale[:, :rows].T.int() - 127
    return torch.ldexp(data.float().view(rows, -1, BLOCK), e[:, :, None]).view(rows, -1)


def _plain(st):
    c = st["case"]
    op, dt = c["op"], NAMES[c["dtype"]]
    out = {}
    if op == "rms":
        s = st["r"].float() + st["x"].float()
        # the sum in 64 bits: a scale's border is one float32 value wide
        k = (1.0 / torch.sqrt(s.double().square().mean(1) + EPS)).float()
        y = s * k[:, None] * st["gamma"]
        if c["train"]:
            out["s"], out["stats"] = s.to(dt), k
        if "y" in c["outs"]:
            out["y"] = y.to(dt)
        if "q" in c["outs"]:
            _put_eight(out, "q", y)
    elif op == "rms_grad":
        k, dy = st["stats"][:, None], st["dy"].float()
        h = st["s"].float() * k
        g = dy * st["gamma"]
        dx = st["ds"].float() + k * (g - h * (g * h).mean(1, keepdim=True))
        out["dx"], out["dgamma"] = dx.to(dt), (dy * h).sum(0)
    elif op == "quantize":
        x = st["x"].float()
        if "q" in c["outs"]:
            _put_eight(out, "q", x)
        if "t" in c["outs"]:
            _put_eight(out, "t", x.T)
    elif op == "matmul8":
        v = _values(st["a"]) @ _values(st["b"]).T
        if c["bias"]:
            v = torch.clamp(v + st["bias"], min=0.0)
        out["c"] = v.to(dt)
    else:
        x, w, label = st["x"].float(), st["w"].float(), st["label"].long()[:, None]
        z = x @ w.T + st["bias"]
        top = z.amax(1, keepdim=True)
        lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
        has = label >= 0
        at = label.clamp(min=0)
        out["loss"] = torch.where(has, lse - z.gather(1, at), 0.0)[:, 0]
        out["lse"] = lse[:, 0]
        if op == "loss_step":
            p = torch.exp(z - lse)
            p.scatter_add_(1, at, torch.full_like(lse, -1.0))
            grad = p * torch.where(has, st["dloss"][:, None], 0.0)
            out["dx"], out["dw"] = (grad @ w).to(dt), (grad.T @ x).to(dt)
            out["dbias"] = grad.sum(0)
    return out


# ----------------------------------------------------------------- reference
def _decoded(q, cols):
    """Float64 values of a matrix in 8 bits, from its bits."""
    bits, scale = q[0].view(torch.uint8).long(), q[1].long()
    code = torch.arange(256, device="cuda", dtype=torch.float64)
    e, m = (code % 128).div(8, rounding_mode="floor"), code % 8
    table = torch.where(e > 0, (8 + m) * 2.0 ** (e - 10), m * 2.0 ** -9) * torch.where(code < 128, 1.0, -1.0)
    v = table[bits]
    power = torch.pow(torch.tensor(2.0, dtype=torch.float64, device="cuda"), (scale[:, :v.shape[0]] - 127).double())
    return (v * power.repeat_interleave(BLOCK, 0).T)[:, :cols]


def exact(case, seed):
    """The operators' definitions in float64 (None for what is held in 8 bits)."""
    op = case["op"]
    if op == "quantize" or (op == "rms" and case["outs"] == "q" and not case["train"]):
        return None
    st = _inputs(case, seed)
    f = {k: v.double() for k, v in st.items() if torch.is_tensor(v)}
    if op == "rms":
        s = f["x"] + f["r"]
        k = ((s * s).sum(1) / s.shape[1] + EPS) ** -0.5
        out = {"s": s, "stats": k} if case["train"] else {}
        if "y" in case["outs"]:
            out["y"] = s * f["gamma"] * k[:, None]
        if "q" in case["outs"]:
            out["q"] = out["q_scale"] = None
        return out
    if op == "rms_grad":
        h = f["s"] * f["stats"][:, None]
        g = f["dy"] * f["gamma"]
        c = (g * h).sum(1) / g.shape[1]
        return {"dx": (g - h * c[:, None]) * f["stats"][:, None] + f["ds"], "dgamma": torch.einsum("rc,rc->c", f["dy"], h)}
    if op == "matmul8":
        v = torch.mm(_decoded(st["a"], case["depth"]), _decoded(st["b"], case["depth"]).T)
        return {"c": (v + f["bias"]).relu() if case["bias"] else v}
    rows, n, dim = case["rows"], case["classes"], case["cols"]
    out = {k: torch.empty(rows, dtype=torch.float64, device="cuda") for k in ("loss", "lse")}
    if op == "loss_step":
        out["dx"] = torch.empty((rows, dim), dtype=torch.float64, device="cuda")
        out["dw"] = torch.zeros((n, dim), dtype=torch.float64, device="cuda")
        out["dbias"] = torch.zeros(n, dtype=torch.float64, device="cuda")
    for r0 in range(0, rows, 2048):
        r = slice(r0, min(rows, r0 + 2048))
        z = torch.addmm(f["bias"], f["x"][r], f["w"].T)
        lse = torch.logsumexp(z, 1)
        label = st["label"][r].long()
        has = (label >= 0).nonzero()[:, 0]
        out["lse"][r] = lse
        loss = torch.zeros_like(lse)
        loss[has] = lse[has] - z[has, label[has]]
        out["loss"][r] = loss
        if op == "loss_step":
            z = z.sub_(lse[:, None]).exp_()
            z[has, label[has]] -= 1.0
            z *= (f["dloss"][r] * (label >= 0))[:, None]
            out["dx"][r] = z @ f["w"]
            out["dw"] += z.T @ f["x"][r]
            out["dbias"] += z.sum(0)
    return out


# ---------------------------------------------------------------------- work
def work(case):
    """Bytes: each input and output once.  Operations: a product's two per term
    (the head's gradients take two more products of the logits' size); per
    element of the norm 4 (addition, square, two multiplications) and 3 more for
    8 bits (magnitude, scaling, rounding), of its backward pass 10 (h, g, the row's
    sum 2, dx 4, the column's sum 2), of a matrix in 8 bits 3 for each form."""
    op, rows, cols = case["op"], case["rows"], case["cols"]
    e = 4 if case["dtype"] == "f32" else 2
    el = rows * cols
    eight = lambda n, k: n * k + n * -(-k // BLOCK)  # noqa: E731
    if op == "rms":
        nbytes = 2 * el * e + 4 * cols + ("y" in case["outs"]) * el * e + ("q" in case["outs"]) * eight(rows, cols)
        return {"bytes": nbytes + case["train"] * (el * e + 4 * rows), "flops": el * (4 + 3 * ("q" in case["outs"]))}
    if op == "rms_grad":
        return {"bytes": 4 * el * e + 4 * rows + 8 * cols, "flops": 10 * el}
    if op == "quantize":
        nbytes = el * e + ("q" in case["outs"]) * eight(rows, cols) + ("t" in case["outs"]) * eight(cols, rows)
        return {"bytes": nbytes, "flops": 3 * el * len(case["outs"])}
    if op == "matmul8":
        k = case["depth"]
        return {"bytes": eight(rows, k) + eight(cols, k) + el * e + 4 * cols * case["bias"], "flops": 2 * el * k}
    n = case["classes"]
    nbytes = (el + n * cols) * e + 4 * n + 12 * rows
    if op == "loss":
        return {"bytes": nbytes, "flops": 2 * el * n}
    return {"bytes": nbytes + (el + n * cols) * e + 4 * n + 4 * rows, "flops": 6 * el * n}
