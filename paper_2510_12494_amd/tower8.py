"""A residual tower whose products take operands in 8 bits, and a head with many
classes, built from the library's operators: for programs that train a party
model of their own, as ``tower``'s, at half the bytes and twice the rate of a
product in bf16, and whose label is one of many items instead of a bit.

    s_0 = x W_in^T                          y_0 = rms norm(s_0)
    h_l = relu(y_l W1_l^T + b_l)
    s_{l+1} = s_l + h_l W2_l^T              y_{l+1} = rms norm(s_{l+1})

and the embedding is the last y, in bf16.  Every product is a vfl_matmul8 of
operands in 8 bits with a power of two for each block of 128: the norms give y
both in 8 bits and in bf16 (vfl_rmsnorm_forward), everything else is converted by
vfl_quantize, which also makes the transposes that the gradients' products read.
Weight gradients are float32; parameters are float32 masters with copies in 8
bits both ways.  Buffers and call descriptors are made once, for at most
``max_rows`` rows.

``ClassHead`` is the label party's loss: logits of ``classes`` items from the
parties' joined embeddings, softmax cross-entropy and its gradients
(vfl_softmax_loss_*), without the logits in memory.
"""
from __future__ import annotations

import torch

from . import vfl as V

EPS = 2.0 ** -17


def _up(n: int, by: int) -> int:
    return -(-n // by) * by


def _set(m, t: torch.Tensor):
    # a single row's stride is of no use and may be anything
    m.data, m.ld = t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1]


class Eight:
    """Room for a matrix in 8 bits (vfl_q8) of at most rows x cols."""

    def __init__(self, rows: int, cols: int, device):
        self.data = torch.empty((rows, _up(cols, V.VFL_Q8_BLOCK)), dtype=torch.uint8, device=device)
        self.scale = torch.empty((_up(cols, V.VFL_Q8_BLOCK) // V.VFL_Q8_BLOCK, _up(rows, 16)), dtype=torch.uint8,
                                 device=device)

    def put(self, m):
        m.data, m.ld, m.scale, m.scale_ld = (self.data.data_ptr(), self.data.stride(0), self.scale.data_ptr(),
                                             self.scale.stride(0))

    def values(self, rows: int, cols: int) -> torch.Tensor:
        """What it stands for, in float64."""
        # 2^e by its bits: a device's pow is not exact
        power = ((self.scale[:, :rows].T.long() - 127 + 1023) << 52).view(torch.float64)
        v = self.data[:rows].view(torch.float8_e4m3fn).double()
        return (v * power.repeat_interleave(V.VFL_Q8_BLOCK, 1))[:, :cols]


def _rows_apart(t: torch.Tensor) -> bool:
    # a stride of 0 would stand for contiguous rows
    return t.stride(1) == 1 and (t.shape[0] == 1 or t.stride(0) >= t.shape[1])


class _Room:
    """Device memory that calls may use one after another.  What a size outgrows stays:
    a captured graph may hold it."""

    def __init__(self, size: int, device):
        self.all = [torch.empty(max(size, 1), dtype=torch.uint8, device=device)]

    def put(self, a, size: int):
        if size > self.all[-1].numel():
            self.all.append(torch.empty(size, dtype=torch.uint8, device=self.all[-1].device))
        a.workspace, a.workspace_bytes = self.all[-1].data_ptr(), self.all[-1].numel()


def _device(device):
    d = torch.device(device)
    return d if d.index is not None else torch.device(d.type, torch.cuda.current_device())


class EightTower:
    """``params`` holds the float32 masters by name (W_in, W1.0, b.0, W2.0,
    gamma.0, ...); ``grads`` their gradients after ``backward``."""

    def __init__(self, d_in: int, width: int, hidden: int, blocks: int, max_rows: int, seed: int = 0,
                 device: str = "cuda:0"):
        self.d_in, self.width, self.hidden, self.blocks, self.max_rows = d_in, width, hidden, blocks, max_rows
        self.dev = _device(device)
        self.trained = 0                                # rows whose training forward the buffers hold
        g = torch.Generator().manual_seed(seed)

        def uniform(n, k):
            return ((torch.rand(n, k, generator=g) * 2 - 1) / k ** 0.5).to(self.dev)

        P = {"W_in": uniform(width, d_in)}
        for l in range(blocks):
            P[f"W1.{l}"], P[f"W2.{l}"] = uniform(hidden, width), uniform(width, hidden)
            P[f"b.{l}"] = torch.zeros(hidden, device=self.dev)
        for l in range(blocks + 1):
            P[f"gamma.{l}"] = torch.ones(width, device=self.dev)
        self.params = P
        self.grads = {k: torch.zeros_like(v) for k, v in P.items()}
        # weights in 8 bits, as they are and transposed (the input gradient's operand)
        self.W = {k: Eight(*v.shape, self.dev) for k, v in P.items() if k.startswith("W")}
        self.WT = {k: Eight(v.shape[1], v.shape[0], self.dev) for k, v in P.items() if k.startswith(("W1", "W2"))}

        new = lambda n: torch.empty((max_rows, n), dtype=torch.bfloat16, device=self.dev)  # noqa: E731
        rows8 = lambda n: Eight(max_rows, n, self.dev)      # noqa: E731
        cols8 = lambda n: Eight(n, max_rows, self.dev)      # noqa: E731
        self.s = [new(width) for _ in range(blocks + 1)]
        self.y = [new(width) for _ in range(blocks + 1)]
        self.h = [new(hidden) for _ in range(blocks)]
        self.branch, self.dh, self.dy = new(width), new(hidden), new(width)
        self.ds = [new(width) for _ in range(2)]
        self.xq, self.yq, self.hq = rows8(d_in), rows8(width), rows8(hidden)
        self.dq = {width: rows8(width), hidden: rows8(hidden)}                       # gradients in 8 bits
        self.turned = {n: (cols8(n), cols8(n)) for n in {width, hidden}}             # and both operands of a weight's
        self.xt = cols8(d_in)               # a training forward's input, for the gradient of W_in
        self.stats = torch.empty((blocks + 1, max_rows), device=self.dev)
        sizes = [(max_rows, width, d_in), (max_rows, hidden, width), (max_rows, width, hidden), (width, hidden, max_rows),
                 (hidden, width, max_rows), (width, d_in, max_rows)]
        # a product of fewer rows may be cut into more parts: room for each power of two below
        need = [V.vfl_norm_workspace_size(max_rows, width)]
        for m, n, k in sizes:
            for r in {max_rows} | {1 << i for i in range(max_rows.bit_length())}:
                need.append(V.vfl_matmul8_workspace_size(r if m == max_rows else m, n, r if k == max_rows else k))
        need += [V.vfl_norm_workspace_size(max_rows, min(hidden, V.VFL_NORM_MAX_COLS))]
        self.ws = _Room(max(need), self.dev)
        self.no_stats = torch.zeros((max_rows, 2), device=self.dev)
        self.refresh()

    # --------------------------------------------------------------- the calls
    def _quantize(self, t: torch.Tensor, q: Eight | None, qt: Eight | None, st: int):
        a = V.vfl_quantize_args()
        a.dtype = V.VFL_BF16 if t.dtype == torch.bfloat16 else V.VFL_F32
        a.rows, a.cols = t.shape
        _set(a.x, t)
        if q is not None:
            q.put(a.q)
        if qt is not None:
            qt.put(a.qt)
        V.vfl_quantize(a, st)

    def _product(self, a8: Eight, b8: Eight, m: int, n: int, k: int, c: torch.Tensor, st: int, bias=None, relu=False):
        a = V.vfl_matmul8_args()
        a.dtype = V.VFL_BF16 if c.dtype == torch.bfloat16 else V.VFL_F32
        a.m, a.n, a.k, a.relu = m, n, k, int(relu)
        a8.put(a.a)
        b8.put(a.b)
        _set(a.c, c)
        if bias is not None:
            a.bias = bias.data_ptr()
        self.ws.put(a, V.vfl_matmul8_workspace_size(m, n, k))
        V.vfl_matmul8(a, st)

    def _norm(self, l: int, rows: int, x: torch.Tensor, r: torch.Tensor | None, s: torch.Tensor | None, st: int):
        a = V.vfl_rmsnorm_args()
        a.dtype, a.rows, a.cols, a.eps = V.VFL_BF16, rows, self.width, EPS
        a.gamma, a.stats = self.params[f"gamma.{l}"].data_ptr(), self.stats[l].data_ptr()
        _set(a.x, x[:rows])
        if r is not None:
            _set(a.r, r[:rows])
            _set(a.s, s[:rows])
        _set(a.y, self.y[l][:rows])
        self.yq.put(a.q)
        V.vfl_rmsnorm_forward(a, st)

    def _norm_backward(self, l: int, rows: int, dy: torch.Tensor, ds: torch.Tensor | None, dx: torch.Tensor, st: int):
        a = V.vfl_rmsnorm_args()
        a.dtype, a.rows, a.cols, a.eps = V.VFL_BF16, rows, self.width, EPS
        a.gamma, a.stats = self.params[f"gamma.{l}"].data_ptr(), self.stats[l].data_ptr()
        a.dgamma = self.grads[f"gamma.{l}"].data_ptr()
        _set(a.s, self.s[l][:rows])
        _set(a.dy, dy[:rows])
        if ds is not None:
            _set(a.ds, ds[:rows])
        _set(a.dx, dx[:rows])
        self.ws.put(a, V.vfl_norm_workspace_size(rows, self.width))
        V.vfl_rmsnorm_backward(a, st)

    def _weight_grad(self, d: torch.Tensor, x: torch.Tensor | Eight, name: str, st: int):
        """d^T x: both operands' blocks run along the rows; x may be there in 8 bits."""
        (n, k), rows = self.grads[name].shape, d.shape[0]
        a8, b8 = self.turned[n][0], x if isinstance(x, Eight) else self.turned[k][1]
        self._quantize(d, None, a8, st)
        if b8 is not x:
            self._quantize(x, None, b8, st)
        self._product(a8, b8, n, k, rows, self.grads[name], st)

    def _column_sums(self, d: torch.Tensor, out: torch.Tensor, st: int):
        """The sum of d over its rows: a layer norm's dbeta, in an order that the sizes
        fix."""
        for c in range(0, d.shape[1], V.VFL_NORM_MAX_COLS):
            part = d[:, c:c + V.VFL_NORM_MAX_COLS]
            a = V.vfl_layernorm_args()
            a.dtype, (a.rows, a.cols), a.eps = V.VFL_BF16, part.shape, EPS
            for m in (a.x, a.dy):
                m.data, m.ld = part.data_ptr(), d.shape[1]
            a.stats, a.dbeta = self.no_stats.data_ptr(), out[c:].data_ptr()
            self.ws.put(a, V.vfl_norm_workspace_size(a.rows, a.cols))
            V.vfl_layernorm_backward(a, st)

    def refresh(self):
        """Rewrite the copies in 8 bits from the masters."""
        with torch.cuda.device(self.dev):
            st = torch.cuda.current_stream(self.dev).cuda_stream
            for k, q in self.W.items():
                self._quantize(self.params[k], q, self.WT.get(k), st)

    @torch.no_grad()
    def forward(self, x: torch.Tensor, train: bool = True) -> torch.Tensor:
        """The embedding of rows ``x`` (bf16), a view of the tower's buffer that the
        next forward overwrites.  Only a training forward can be followed by
        ``backward``, which takes nothing more from x: its owner may use it again."""
        if (x.dim() != 2 or not 1 <= x.shape[0] <= self.max_rows or x.shape[1] != self.d_in
                or x.dtype != torch.bfloat16 or x.device != self.dev or not _rows_apart(x)):
            raise ValueError(f"x must be [1..{self.max_rows} x {self.d_in}] of bfloat16 on {self.dev}, rows apart")
        rows, W = x.shape[0], self.W
        self.trained = 0
        with torch.cuda.device(self.dev):
            st = torch.cuda.current_stream(self.dev).cuda_stream
            self._quantize(x, self.xq, self.xt if train else None, st)
            self._product(self.xq, W["W_in"], rows, self.width, self.d_in, self.s[0][:rows], st)
            self._norm(0, rows, self.s[0], None, None, st)
            for l in range(self.blocks):
                h = self.h[l][:rows]
                self._product(self.yq, W[f"W1.{l}"], rows, self.hidden, self.width, h, st, self.params[f"b.{l}"], True)
                self._quantize(h, self.hq, None, st)
                self._product(self.hq, W[f"W2.{l}"], rows, self.width, self.hidden, self.branch[:rows], st)
                self._norm(l + 1, rows, self.branch, self.s[l], self.s[l + 1], st)
        if train:
            self.trained = rows
        return self.y[self.blocks][:rows]

    @torch.no_grad()
    def backward(self, dz: torch.Tensor):
        """Gradients of every parameter into ``grads`` for the gradient ``dz`` of
        the last forward's embedding, which has to be a training one."""
        if not self.trained or dz.shape != (self.trained, self.width) or dz.device != self.dev:
            raise ValueError(f"dz must be [{self.trained} x {self.width}] on {self.dev}, of a training forward's rows")
        rows, G = dz.shape[0], self.grads
        with torch.cuda.device(self.dev):
            st = torch.cuda.current_stream(self.dev).cuda_stream
            dy = dz.to(torch.bfloat16).contiguous()
            ds, other = self.ds
            self._norm_backward(self.blocks, rows, dy, None, ds, st)
            for l in reversed(range(self.blocks)):
                d, h, dh = ds[:rows], self.h[l][:rows], self.dh[:rows]
                self._weight_grad(d, h, f"W2.{l}", st)
                self._quantize(d, self.dq[self.width], None, st)
                self._product(self.dq[self.width], self.WT[f"W2.{l}"], rows, self.hidden, self.width, dh, st)
                dh.masked_fill_(h <= 0, 0.0)       # whatever it holds: a product would leave NaN of an infinity
                self._column_sums(dh, G[f"b.{l}"], st)
                self._weight_grad(dh, self.y[l][:rows], f"W1.{l}", st)
                self._quantize(dh, self.dq[self.hidden], None, st)
                self._product(self.dq[self.hidden], self.WT[f"W1.{l}"], rows, self.width, self.hidden, self.dy[:rows], st)
                self._norm_backward(l, rows, self.dy, ds, other, st)
                ds, other = other, ds
            self._weight_grad(ds[:rows], self.xt, "W_in", st)

    @torch.no_grad()
    def sgd(self, lr: float):
        for k, v in self.params.items():
            v.add_(self.grads[k], alpha=-lr)
        self.refresh()


class ClassHead:
    """A linear head with a softmax cross-entropy over ``classes`` items: float32
    masters ``W`` [classes x dim] and ``bias``, a copy of W in bf16, gradients
    ``dW`` (bf16) and ``dbias`` after ``loss``."""

    def __init__(self, dim: int, classes: int, max_rows: int, seed: int = 0, device: str = "cuda:0"):
        self.dim, self.classes, self.max_rows = dim, classes, max_rows
        self.dev = _device(device)
        g = torch.Generator().manual_seed(seed)
        self.W = ((torch.rand(classes, dim, generator=g) * 2 - 1) / dim ** 0.5).to(self.dev)
        self.bias = torch.zeros(classes, device=self.dev)
        self.copy, self.dW = self.W.bfloat16(), torch.empty_like(self.W, dtype=torch.bfloat16)
        self.dbias = torch.empty_like(self.bias)
        self.losses, self.lse = (torch.empty(max_rows, device=self.dev) for _ in range(2))
        self.dz = torch.empty((max_rows, dim), dtype=torch.bfloat16, device=self.dev)
        self.ws = _Room(V.vfl_softmax_loss_workspace_size(V.VFL_BF16, max_rows, dim, classes), self.dev)

    @torch.no_grad()
    def loss(self, z: torch.Tensor, labels: torch.Tensor, train: bool = True):
        """The rows' losses for embeddings ``z`` (bf16) and int32 ``labels`` (outside
        the classes: a row without one), and the gradient of their mean over the
        rows with respect to z (None without ``train``): views that the next call overwrites."""
        if (z.dim() != 2 or not 1 <= z.shape[0] <= self.max_rows or z.shape[1] != self.dim or z.dtype != torch.bfloat16
                or z.device != self.dev or not _rows_apart(z)):
            raise ValueError(f"z must be [1..{self.max_rows} x {self.dim}] of bfloat16 on {self.dev}, rows apart")
        rows = z.shape[0]
        if labels.shape != (rows,) or labels.dtype != torch.int32 or labels.device != self.dev or not labels.is_contiguous():
            raise ValueError(f"labels must be {rows} contiguous int32 values on {self.dev}")
        with torch.cuda.device(self.dev):
            st = torch.cuda.current_stream(self.dev).cuda_stream
            a = V.vfl_softmax_loss_args()
            a.dtype, a.rows, a.dim, a.classes, a.scale = V.VFL_BF16, rows, self.dim, self.classes, 1.0 / rows
            for m, t in ((a.x, z), (a.w, self.copy), (a.dx, self.dz[:rows]), (a.dw, self.dW)):
                _set(m, t)
            a.bias, a.labels, a.loss, a.lse, a.dbias = (t.data_ptr() for t in (self.bias, labels, self.losses, self.lse,
                                                                              self.dbias))
            self.ws.put(a, V.vfl_softmax_loss_workspace_size(V.VFL_BF16, rows, self.dim, self.classes))
            V.vfl_softmax_loss_forward(a, st)
            if train:
                V.vfl_softmax_loss_backward(a, st)
        return self.losses[:rows], self.dz[:rows] if train else None

    @torch.no_grad()
    def sgd(self, lr: float):
        self.W.add_(self.dW, alpha=-lr)
        self.bias.add_(self.dbias, alpha=-lr)
        self.copy.copy_(self.W)
