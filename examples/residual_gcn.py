"""Trains a GCN of several layers on nodes that carry an id only (lookup, root-mean-square norms around a residual, aggregation over a HAG, SoftMax loss, AdamW with clipping and states in 8
bits), then serves it with its matrices and normed rows in 8 bits.

    python examples/residual_gcn.py [--blocks 16] [--block 64] [--d 64] [--layers 3] [--steps 60] [--lr 0.01] [--max-norm 1.0] [--bits 8]

The graph is a stochastic block model and a node's class is its block; half of the nodes have a label, the others are what the accuracies are taken of.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1906_03707_amd import binding, layers, synth  # noqa: E402


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--blocks", type=int, default=16)
    ap.add_argument("--block", type=int, default=64)
    ap.add_argument("--d", type=int, default=64)
    ap.add_argument("--layers", type=int, default=3)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=0.01)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args(argv)
    rowptr, col = synth.sbm(a.blocks, a.block, 0.2, 0.002, seed=1)
    n, classes = rowptr.size - 1, (a.blocks + 3) // 4 * 4
    h = binding.hag_search(rowptr, col, n // 4).upload()
    gen = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *shape: (shape[-2] ** -0.5 * torch.randn(*shape, generator=gen, device="cuda")).requires_grad_()   # noqa: E731
    ones = lambda: torch.ones(a.d, device="cuda", requires_grad=True)   # noqa: E731
    table = (a.d ** -0.5 * torch.randn(n, a.d, generator=gen, device="cuda")).requires_grad_()
    params = [table] + [p for _ in range(a.layers) for p in (ones(), normal(a.d, a.d))] + [ones(), normal(a.d, classes)]
    optimizer = layers.AdamW(params, lr=a.lr, bits=a.bits)
    ids = torch.arange(n, device="cuda")
    truth = torch.from_numpy(np.repeat(np.arange(a.blocks), a.block)).cuda()
    known = torch.rand(n, generator=gen, device="cuda") < 0.5
    labels = torch.where(known, truth, -100)
    for step in range(a.steps):
        loss, norm = layers.residual_gcn_step(h, ids, params, labels, optimizer, a.max_norm)
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {loss.item():.4f}, gradient norm {norm.item():.3f}", flush=True)
    with torch.no_grad():
        logits = layers.residual_gcn_logits(h, ids, params)
    served = layers.residual_gcn_logits_fp8(h, ids, layers.residual_gcn_fp8(params))
    accuracies = [(z.argmax(1) == truth)[~known].float().mean().item() for z in (logits, served)]
    print(f"accuracy on the {int((~known).sum())} nodes without a label: {accuracies[0]:.3f}, served in 8 bits {accuracies[1]:.3f}")
    return loss.item(), *accuracies


if __name__ == "__main__":
    main()
