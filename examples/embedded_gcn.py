"""Trains a 2-layer GCN on a graph whose nodes have no features, only an id each: a table of rows that is learnt with the weights (lookup, layer norm,
aggregation over a HAG, SoftMax loss, clipped gradients).

    python examples/embedded_gcn.py [--blocks 16] [--block 64] [--d 64] [--steps 60] [--lr 2.0] [--max-norm 1.0]

The graph is a stochastic block model and a node's class is its block; half of the nodes have a label, the others are what the accuracy is taken of.
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
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=2.0)
    ap.add_argument("--max-norm", type=float, default=1.0)
    a = ap.parse_args(argv)
    rowptr, col = synth.sbm(a.blocks, a.block, 0.2, 0.002, seed=1)
    n, classes = rowptr.size - 1, (a.blocks + 3) // 4 * 4
    h = binding.hag_search(rowptr, col, n // 4).upload()
    gen = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *shape, std: (std * torch.randn(*shape, generator=gen, device="cuda")).requires_grad_()   # noqa: E731
    params = (normal(n, a.d, std=a.d ** -0.5), torch.ones(a.d, device="cuda", requires_grad=True), torch.zeros(a.d, device="cuda", requires_grad=True),
              normal(a.d, 16, std=a.d ** -0.5), normal(16, classes, std=0.25))
    ids = torch.arange(n, device="cuda")
    truth = torch.from_numpy(np.repeat(np.arange(a.blocks), a.block)).cuda()
    known = torch.rand(n, generator=gen, device="cuda") < 0.5
    labels = torch.where(known, truth, -100)
    for step in range(a.steps):
        loss, norm = layers.embedded_gcn2_step(h, ids, params, labels, a.lr, a.max_norm)
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {loss.item():.4f}, gradient norm {norm.item():.3f}", flush=True)
    with torch.no_grad():
        table, w, b, w1, w2 = params
        agg = layers.aggregation(h, "gcn")
        x = layers.layer_norm(layers.embedding(table, ids, a.d ** 0.5), w, b)
        logits = agg(torch.relu(agg(x @ w1)) @ w2)
        accuracy = (logits.argmax(1) == truth)[~known].float().mean().item()
    print(f"accuracy on the {int((~known).sum())} nodes without a label: {accuracy:.3f}")
    return loss.item(), accuracy


if __name__ == "__main__":
    main()
