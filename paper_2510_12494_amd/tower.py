"""A residual tower, built from the library's row operators: an alternative to
the plain bottom MLP of ``session`` for programs that train a party model of
their own and hand its embeddings and their gradients over themselves.

    s_0 = x W_in^T                       y_0 = layer norm(s_0)
    a_l = dropout(relu(y_l W1_l^T + b_l))
    s_{l+1} = s_l + dropout(a_l W2_l^T)  y_{l+1} = layer norm(s_{l+1})

and the embedding is the last y.  The dropouts, norms and joins run in the
library's kernels (vfl_dropout, vfl_layernorm_*, vfl_residual_*), the products
in torch's matmul, whose results have the tower's dtype; weight gradients are
float32, unrounded.  Parameters are float32 masters with operand copies in the
tower's dtype, as in the library's own models; buffers and call descriptors are
made once, for at most ``max_rows`` rows.  A dropout mask follows from (seed,
step, layer, sample id), so the backward pass stores none and a sample's mask
does not depend on how the batch is split.
"""
from __future__ import annotations

import torch

from . import vfl as V

EPS = 1e-5


def _set(m, t: torch.Tensor):
    # a single row's stride is of no use and may be anything
    m.data, m.ld = t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1]


class ResidualTower:
    """``params`` holds the float32 masters by name (W_in, W1.0, b.0, W2.0,
    gamma.0, beta.0, ...); ``grads`` their gradients after ``backward``."""

    def __init__(self, d_in: int, width: int, hidden: int, blocks: int, max_rows: int, dtype: str = "bf16",
                 p: float = 0.1, seed: int = 0, device: str = "cuda:0"):
        self.d_in, self.width, self.hidden, self.blocks, self.max_rows = d_in, width, hidden, blocks, max_rows
        self.p, self.seed = p, seed
        if dtype not in ("bf16", "f32"):
            raise ValueError(f"dtype must be 'bf16' or 'f32', not {dtype!r}")
        dev = torch.device(device)
        self.dev = dev if dev.index is not None else torch.device(dev.type, torch.cuda.current_device())
        self.bf16, self.trained = dtype == "bf16", 0        # rows whose training forward the buffers hold
        self.next_step = 0                                  # of a training forward that names none
        self.tdt = torch.bfloat16 if self.bf16 else torch.float32
        g = torch.Generator().manual_seed(seed)

        def uniform(n, k):
            return ((torch.rand(n, k, generator=g) * 2 - 1) / k ** 0.5).to(self.dev)

        P = {"W_in": uniform(width, d_in)}
        for l in range(blocks):
            P[f"W1.{l}"], P[f"W2.{l}"] = uniform(hidden, width), uniform(width, hidden)
            P[f"b.{l}"] = torch.zeros(hidden, device=self.dev)
        for l in range(blocks + 1):
            P[f"gamma.{l}"] = torch.ones(width, device=self.dev)
            P[f"beta.{l}"] = torch.zeros(width, device=self.dev)
        self.params = P
        self.grads = {k: torch.zeros_like(v) for k, v in P.items()}
        self.copies = {k: torch.empty_like(v, dtype=self.tdt) for k, v in P.items() if k.startswith(("W", "b."))}
        self.refresh()

        new = lambda n: torch.empty((max_rows, n), dtype=self.tdt, device=self.dev)  # noqa: E731
        self.s = [new(width) for _ in range(blocks + 1)]
        self.y = [new(width) for _ in range(blocks + 1)]
        self.h = [new(hidden) for _ in range(blocks)]       # relu(...)
        self.a = [new(hidden) for _ in range(blocks)]       # after dropout
        self.branch, self.ds, self.dbranch = new(width), new(width), new(width)
        self.dh = new(hidden)
        self.stats = torch.empty((blocks + 1, max_rows, 2), dtype=torch.float32, device=self.dev)
        self.ws_bytes = V.vfl_norm_workspace_size(max_rows, width)
        self.ws = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=self.dev)
        self._describe()

    def _describe(self):
        code = V.VFL_BF16 if self.bf16 else V.VFL_F32
        self.norm0 = n = V.vfl_layernorm_args()
        _set(n.x, self.s[0])
        _set(n.y, self.y[0])
        self.joins, self.drops, self.undrops = [], [], []
        for l in range(self.blocks):
            j = V.vfl_residual_args()
            _set(j.x, self.branch)
            _set(j.r, self.s[l])
            _set(j.s, self.s[l + 1])
            _set(j.y, self.y[l + 1])
            _set(j.ds, self.ds)                     # dr over ds, dx over its own buffer
            _set(j.dr, self.ds)
            _set(j.dx, self.dbranch)
            j.drop.tag = 2 * l + 1
            self.joins.append(j)
            for src, dst, calls in ((self.h[l], self.a[l], self.drops), (self.dh, self.dh, self.undrops)):
                d = V.vfl_dropout_args()
                _set(d.x, src)
                _set(d.y, dst)
                d.dtype, d.cols = code, self.hidden
                d.drop.tag = 2 * l
                calls.append(d)
        for l, a in enumerate([n, *self.joins]):
            a.dtype, a.cols, a.eps = code, self.width, EPS
            a.gamma, a.beta = self.params[f"gamma.{l}"].data_ptr(), self.params[f"beta.{l}"].data_ptr()
            a.dgamma, a.dbeta = self.grads[f"gamma.{l}"].data_ptr(), self.grads[f"beta.{l}"].data_ptr()
            a.stats = self.stats[l].data_ptr()
            a.workspace, a.workspace_bytes = self.ws.data_ptr(), self.ws_bytes
        for a in [*self.joins, *self.drops, *self.undrops]:
            a.drop.p, a.drop.seed = self.p, self.seed

    def refresh(self):
        """Rewrite the operand copies from the masters."""
        for k, c in self.copies.items():
            c.copy_(self.params[k])

    def _call(self, rows: int, row0: int, step: int, p: float):
        for a in [*self.joins, *self.drops, *self.undrops]:
            a.rows, a.drop.row0, a.drop.step, a.drop.p = rows, row0, step, p
        self.norm0.rows = rows
        return torch.cuda.current_stream(self.dev).cuda_stream

    @torch.no_grad()
    def forward(self, x: torch.Tensor, row0: int = 0, step: int | None = None, train: bool = True) -> torch.Tensor:
        """The embedding of rows ``x`` (global sample ids from ``row0``), a view of
        the tower's buffer that the next forward overwrites; without ``train``
        nothing is dropped (scoring).  ``step`` keys the masks: towers that have to
        make the same ones (replicas, a replay, a batch in parts) name it; without
        it a training forward takes the step after the last one's, from 0."""
        if (x.dim() != 2 or not 1 <= x.shape[0] <= self.max_rows or x.shape[1] != self.d_in or x.dtype != self.tdt
                or x.device != self.dev):
            raise ValueError(f"x must be [1..{self.max_rows} x {self.d_in}] of {self.tdt} on {self.dev}")
        rows, c = x.shape[0], self.copies
        self.trained = 0
        if step is None:
            step = self.next_step
        with torch.cuda.device(self.dev):
            st = self._call(rows, row0, step, self.p if train else 0.0)
            self.x = x
            torch.matmul(x, c["W_in"].T, out=self.s[0][:rows])
            V.vfl_layernorm_forward(self.norm0, st)
            for l in range(self.blocks):
                h, a = self.h[l][:rows], self.a[l][:rows]
                torch.addmm(c[f"b.{l}"], self.y[l][:rows], c[f"W1.{l}"].T, out=h)
                h.relu_()
                V.vfl_dropout(self.drops[l], st)
                torch.matmul(a, c[f"W2.{l}"].T, out=self.branch[:rows])
                V.vfl_residual_forward(self.joins[l], st)
        if train:
            self.trained, self.next_step = rows, step + 1
        return self.y[self.blocks][:rows]

    def _weight_grad(self, d: torch.Tensor, x: torch.Tensor, out: torch.Tensor):
        if self.bf16:
            torch.mm(d.T, x, out_dtype=torch.float32, out=out)
        else:
            torch.mm(d.T, x, out=out)

    @torch.no_grad()
    def backward(self, dz: torch.Tensor):
        """Gradients of every parameter into ``grads`` for the gradient ``dz`` of
        the last forward's embedding, which has to be a training one."""
        if not self.trained or dz.shape != (self.trained, self.width) or dz.device != self.dev:
            raise ValueError(f"dz must be [{self.trained} x {self.width}] on {self.dev}, of a training forward's rows")
        rows, G, c = dz.shape[0], self.grads, self.copies
        with torch.cuda.device(self.dev):
            st = torch.cuda.current_stream(self.dev).cuda_stream
            dy = dz.to(self.tdt).contiguous()
            ds = self.ds[:rows].zero_()
            for l in reversed(range(self.blocks)):
                j = self.joins[l]
                _set(j.dy, dy)
                V.vfl_residual_backward(j, st)
                db, dh = self.dbranch[:rows], self.dh[:rows]
                self._weight_grad(db, self.a[l][:rows], G[f"W2.{l}"])
                torch.matmul(db, c[f"W2.{l}"], out=dh)
                V.vfl_dropout(self.undrops[l], st)
                dh.mul_(self.h[l][:rows] > 0)
                self._weight_grad(dh, self.y[l][:rows], G[f"W1.{l}"])
                torch.sum(dh, 0, dtype=torch.float32, out=G[f"b.{l}"])
                dy = torch.matmul(dh, c[f"W1.{l}"])
            n = self.norm0
            _set(n.dy, dy)
            _set(n.dx, self.dbranch)
            V.vfl_layernorm_backward(n, st)
            ds += self.dbranch[:rows]
            self._weight_grad(ds, self.x, G["W_in"])

    @torch.no_grad()
    def sgd(self, lr: float):
        for k, v in self.params.items():
            v.add_(self.grads[k], alpha=-lr)
        self.refresh()
