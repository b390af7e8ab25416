"""Adapters of several requests beside one pruned layer: trained together by the AdamW step, then answering.

The layer is pruned and rounded to bfloat16 once (condensa_prune) and stays as it is.  Every request has a low-rank adapter of its own; the
forward and backward passes take the tokens of all requests at once, and one AdamW launch updates all adapters, with states in 8 bits and
the weights' bfloat16 copies, which the next forward pass reads, written by the same launch.  At the end a token of each request is answered.

    python examples/adapters.py [--steps 200]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_1911_02497_amd as P  # noqa: E402

N_IN, N_OUT, RANK, REQUESTS, TOKENS = 512, 2048, 8, 4, 128


def run(steps, dev="cuda"):
    """Mean square errors of the adapted layer against its targets: before the first step, after the last, and of the single tokens."""
    g = torch.Generator(dev).manual_seed(7)
    normal = lambda std, *shape: torch.randn(*shape, device=dev, generator=g) * std  # noqa: E731
    dense = normal(0.04, N_OUT, N_IN)
    theta = P.condensa_prune([dense], [0.5], theta=True, mask=False)["theta"][0][0]
    w = theta.view(N_OUT, N_IN).bfloat16()

    # master weights in binary32, their copies that the products read, gradients, and states in 8 bits
    master = [t for _ in range(REQUESTS) for t in (normal(N_IN ** -0.5, RANK, N_IN), torch.zeros(N_OUT, RANK, device=dev))]
    copies = [t.bfloat16() for t in master]
    grads = [torch.zeros_like(t) for t in master]
    codes = [[torch.zeros(t.shape, dtype=torch.uint8, device=dev) for t in master] for _ in range(2)]
    scales = [[torch.zeros(-(-t.numel() // P.STATE_BLOCK), device=dev) for t in master] for _ in range(2)]
    pairs = lambda ts: list(zip(ts[0::2], ts[1::2]))  # noqa: E731
    adapters = P.adapter_table([(a, b, 1.0) for a, b in pairs(copies)], grads=pairs(grads))
    adamw = P.adamw_table(master, grads, *codes, exp_avg_scale=scales[0], exp_avg_sq_scale=scales[1], codes=copies)

    # every request wants the dense layer with a shift of its own
    x = normal(1.0, TOKENS, N_IN).bfloat16()
    ids = (torch.arange(TOKENS, device=dev) * REQUESTS // TOKENS).to(torch.int32)
    shift = [normal(0.02, N_OUT, 4) @ normal(0.2, 4, N_IN) for _ in range(REQUESTS)]
    target = torch.cat([x[ids == r].float() @ (w.float() + shift[r]).t() for r in range(REQUESTS)])

    z = torch.empty(TOKENS, RANK, device=dev, dtype=torch.bfloat16)
    forward, backward = P.adapter_workspace(adapters, TOKENS), P.adapter_workspace(adapters, TOKENS, backward=True)
    losses = []
    for step in range(1, steps + 1):
        y = P.condensa_adapter_project(x, w, adapters, ids, z=z, workspace=forward)["y"]
        error = y.float() - target
        losses.append(error.square().mean())
        dy = (error * (2 / error.numel()) * 2.0 ** 10).bfloat16()                # scaled up for the 16-bit type, and back in the step
        P.condensa_adapter_project_backward(dy, x, w, adapters, ids, z, dx=False, workspace=backward)
        P.condensa_lc_adamw_step(adamw, 5e-3, step, seed=step * 0x9E3779B97F4A7C15, grad_scale=torch.full((1,), 2.0 ** -10, device=dev))
    one = torch.arange(0, TOKENS, TOKENS // REQUESTS, device=dev)
    answer = P.condensa_adapter_project(x[one], w, adapters, ids[one])["y"]
    return float(losses[0]), float(losses[-1]), float((answer.float() - target[one]).square().mean())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    print("mean square error: %.4g before, %.4g after training, %.4g of single tokens" % run(ap.parse_args().steps))
