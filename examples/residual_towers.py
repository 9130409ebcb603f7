"""Two-party split training with residual towers in place of plain MLP bottoms.

Each party runs a tower of residual blocks (layer norm, dropout, residual join:
the library's row operators) on its own features; party B's embedding goes to
party A, which holds the labels, a linear head on both embeddings and the
binary cross-entropy, and sends back the gradient of B's embedding.  Both run in
one process and hand these over as tensors, in step (the library's channels,
with their bounded staleness, clipping and noise, carry the messages of its own
bottom models).  Synthetic data (the seeded teacher of vfl_synth), plain SGD.

    python examples/residual_towers.py [--steps 200] [--rows 20000] [--dtype bf16]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import vfl_synth as S  # noqa: E402
from paper_2510_12494_amd.tower import ResidualTower  # noqa: E402


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--rows", type=int, default=20_000)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=3)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--lr", type=float, default=0.1)
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    args = ap.parse_args(argv)

    w = S.get("dense_tabular").with_rows(args.rows)
    data = S.generate(w, args.rows)
    tdt = torch.bfloat16 if args.dtype == "bf16" else torch.float32
    xa, xb = (torch.from_numpy(data[k]).to("cuda", tdt) for k in ("xa", "xb"))
    y = torch.from_numpy(data["y"]).cuda()

    tower = lambda x, seed: ResidualTower(x.shape[1], args.width, args.width, args.blocks, args.batch,  # noqa: E731
                                          args.dtype, args.dropout, seed)
    A, B = tower(xa, 11), tower(xb, 12)
    head = torch.zeros(2 * args.width, device="cuda")
    bias = torch.zeros(1, device="cuda")

    losses = []
    per_epoch = -(-args.rows // args.batch)
    for t in range(args.steps):
        r0 = t % per_epoch * args.batch
        rows = slice(r0, min(r0 + args.batch, args.rows))      # the last batch of an epoch is short
        z = torch.cat([A.forward(xa[rows], r0, t), B.forward(xb[rows], r0, t)], 1).float()
        logit = z @ head + bias
        losses.append(torch.nn.functional.binary_cross_entropy_with_logits(logit, y[rows]))
        g = (torch.sigmoid(logit) - y[rows]) / len(logit)
        dz = g[:, None] * head
        head -= args.lr * (z.T @ g)
        bias -= args.lr * g.sum()
        for party, d in ((A, dz[:, :args.width]), (B, dz[:, args.width:])):
            party.backward(d)
            party.sgd(args.lr)
        if t % 20 == 0 or t == args.steps - 1:
            print(f"step {t:4d}  loss {losses[-1].item():.4f}", flush=True)

    # score: nothing dropped, one sample at a time as a service would
    hits, n = 0, min(64, args.rows)
    for i in range(n):
        z = torch.cat([A.forward(xa[i:i + 1], i, train=False), B.forward(xb[i:i + 1], i, train=False)], 1).float()
        hits += int((z @ head + bias > 0).item() == bool(y[i].item()))
    print(f"scored {n} samples one by one: {hits / n:.2f} correct")
    return [float(v) for v in losses], hits / n


if __name__ == "__main__":
    main()
