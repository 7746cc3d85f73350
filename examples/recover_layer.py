"""Prune one linear layer and win its answers back: calibrate -> prune 2:4 -> tune the weights that
stay -> train an adapter per task -> serve tokens of all tasks in one call.

    python examples/recover_layer.py [--rows 2048 --cols 2048 --tokens 4096 --tasks 4 --rank 16]

The data is synthetic.  The dense layer W0 is the teacher; task i wants W0 + D_i, D_i of low rank.
Every product with the layer's weights, every gradient and every update runs in the library; torch
makes the data, holds it, and takes the difference of two results.
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2504_05346_b200 as thanos  # noqa: E402


def parse(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rows", type=int, default=2048, help="output features c")
    ap.add_argument("--cols", type=int, default=2048, help="input features b (a multiple of 8)")
    ap.add_argument("--tokens", type=int, default=4096, help="tokens of a calibration or training batch")
    ap.add_argument("--tasks", type=int, default=4)
    ap.add_argument("--rank", type=int, default=16)
    ap.add_argument("--weight-steps", type=int, default=30)
    ap.add_argument("--adapter-steps", type=int, default=40)
    ap.add_argument("--seed", type=int, default=0)
    return ap.parse_args(argv)


def relative(Y, target):
    return ((Y.float() - target.float()).norm() / target.float().norm()).item()


def main(argv=None):
    a = parse(argv)
    c, b, T, n, r = a.rows, a.cols, a.tokens, a.tasks, a.rank
    gen = torch.Generator(device="cuda").manual_seed(a.seed)
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    bf = torch.bfloat16

    # correlated inputs: without correlation there is nothing for the remaining weights to make up
    mix = randn(b, b) / math.sqrt(b) + 0.3 * torch.eye(b, device="cuda")
    tokens = lambda k: (randn(k, b) @ mix).to(bf)  # noqa: E731
    W0 = (randn(c, b) / math.sqrt(b)).to(bf)
    X, held = tokens(T), tokens(1024)
    out = {}

    # ---- calibrate and prune: two of every four columns go
    H = torch.zeros((b, b), device="cuda")
    thanos.hessian_accumulate(H, X)
    factor, xnorm = thanos.prepare_inverse(H.clone(), 0.01)
    W, mask, _ = thanos.prune_layer(W0, factor, xnorm, thanos.NM, n=2, m=4, B=128)
    teacher, _ = thanos.adapter_forward(held, W0)
    out["pruned"] = relative(thanos.adapter_forward(held, W)[0], teacher)

    # ---- tune the weights that stay: the layer's error |X (W - W0)^T|^2 has the gradient (W - W0) H.
    # The mask is part of the step, so the zeros of the 2:4 pattern stay exact zeros.
    master, momentum, dense = W.float(), torch.zeros((c, b), device="cuda"), W0.float()
    for i in range(a.weight_steps):
        G = thanos.dense_product(master - dense, H, check=False)
        thanos.orthogonal_step(master, momentum, G, mask=mask, momentum=0.9,
                               lr=0.02 / math.sqrt(b) * (1 - i / a.weight_steps),
                               gain=math.sqrt(max(1.0, c / b)), W_out=master, M_out=momentum)
    W = master.to(bf)
    assert not W[mask != 0].any()
    out["tuned"] = relative(thanos.adapter_forward(held, W)[0], teacher)

    # ---- train the tasks' adapters together on the frozen pruned weights
    delta = [0.5 / math.sqrt(b) * randn(c, 4) @ randn(4, b) / 2 for _ in range(n)]
    scale = torch.full((n,), 2.0, device="cuda")
    A, B = randn(n, r, b) / math.sqrt(b), torch.zeros((n, c, r), device="cuda")
    mA, mB = torch.zeros_like(A), torch.zeros_like(B)

    def batch(k):
        x = tokens(k)
        task = torch.randint(0, n, (k,), generator=gen, device="cuda", dtype=torch.int32)
        target = thanos.adapter_forward(x, W0)[0].float()
        for i in range(n):
            rows = (task == i).nonzero().squeeze(1)
            target[rows] += x[rows].float() @ delta[i].t()
        return x, task, target.to(bf)

    xt, task_t, want_t = batch(1024)
    out["tasks before"] = relative(thanos.adapter_forward(xt, W)[0], want_t)
    for i in range(a.adapter_steps):
        x, task, want = batch(T)
        lr = 0.1 * (1 - i / a.adapter_steps)
        Ab, Bb = A.to(bf), B.to(bf)
        Y, V = thanos.adapter_forward(x, W, Ab, Bb, task, scale)
        _, dA, dB = thanos.adapter_backward((Y - want) / T, x, V, W, Ab, Bb, task, scale,
                                            need_dx=False)
        thanos.orthogonal_step(A, mA, dA, lr=lr, momentum=0.9, W_out=A, M_out=mA)
        thanos.orthogonal_step(B, mB, dB, lr=lr, momentum=0.9, W_out=B, M_out=mB)
    Ab, Bb = A.to(bf), B.to(bf)
    out["tasks after"] = relative(thanos.adapter_forward(xt, W, Ab, Bb, task_t, scale)[0], want_t)

    # ---- serve: one token a request, the last request without an adapter
    x = held[:n + 1].contiguous()
    who = torch.tensor(list(range(n)) + [-1], dtype=torch.int32, device="cuda")
    together, _ = thanos.adapter_forward(x, W, Ab, Bb, who, scale)
    alone = torch.cat([thanos.adapter_forward(x[t:t + 1], W, Ab, Bb, who[t:t + 1], scale)[0]
                       for t in range(n + 1)])
    out["served together against alone"] = relative(together, alone)
    torch.cuda.synchronize()
    return out


if __name__ == "__main__":
    for name, value in main().items():
        print("%-32s relative error %.4f" % (name, value))
