"""Two-party split training with towers in 8 bits and a label that is one of many
items.

Each party runs a tower whose products take operands in 8 bits on its own
features; party B's embedding goes to party A, which holds the labels (which item a
sample took), a linear head over all items with the softmax cross-entropy, and sends
back the gradient of B's embedding.  Both run in one process and hand these over as
tensors, in step.  Synthetic data: an item is a point in the joint feature space, a
sample one of them with noise.  Plain SGD.

    python examples/eight_bit_towers.py [--steps 200] [--classes 2000]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2510_12494_amd.tower8 import ClassHead, EightTower  # noqa: E402


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--classes", type=int, default=2000)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--lr", type=float, default=1.0)
    args = ap.parse_args(argv)

    g = torch.Generator(device="cuda").manual_seed(7)
    items = torch.randn(args.classes, 96, generator=g, device="cuda")

    def batch(n):
        label = torch.randint(0, args.classes, (n,), generator=g, device="cuda")
        x = (items[label] + 0.5 * torch.randn(n, 96, generator=g, device="cuda")).bfloat16()
        return x[:, :32].contiguous(), x[:, 32:].contiguous(), label.int()

    A = EightTower(32, args.width, args.width, args.blocks, args.batch, seed=1)
    B = EightTower(64, args.width, args.width, args.blocks, args.batch, seed=2)
    head = ClassHead(2 * args.width, args.classes, args.batch, seed=3)
    losses = []
    for t in range(args.steps):
        xa, xb, label = batch(args.batch)
        z = torch.cat([A.forward(xa), B.forward(xb)], 1)
        loss, dz = head.loss(z, label)
        losses.append(loss.mean())
        for party, d in ((A, dz[:, :args.width]), (B, dz[:, args.width:])):
            party.backward(d)
            party.sgd(args.lr)
        head.sgd(args.lr)
        if t % 20 == 0 or t == args.steps - 1:
            print(f"step {t:4d}  loss {losses[-1].item():.4f}", flush=True)

    # score: one sample at a time as a service would
    xa, xb, label = batch(32)
    one = torch.cat([head.loss(torch.cat([A.forward(xa[i:i + 1], train=False), B.forward(xb[i:i + 1], train=False)], 1),
                               label[i:i + 1], train=False)[0].clone() for i in range(32)])
    print(f"scored 32 samples one by one: mean loss {one.mean().item():.4f}")
    return [float(v) for v in losses], float(one.mean())


if __name__ == "__main__":
    main()
