"""A small data-parallel training loop with every call in its place: embedding
lookup, backward pass, embedding gradient, bucketed synchronization, global
norm, AdamW.

    python -m paper_2006_15704_amd.train --replicas 4 --bits 8

The model predicts the next token from the last one: logits = x W^T + b with
x = scale * table[token].  Its tokens follow a fixed random successor nine times out
of ten, so the loss falls from log(vocabulary) towards the entropy of that.
R replicas (the R training processes) draw their own batches; the library averages their
gradients and steps replica 0's parameters, which all replicas read.  The products and the
softmax in between are PyTorch's.
"""
from __future__ import annotations

import argparse
import math
from typing import List

import torch

from . import binding as B
from . import harness

LR, BETA1, BETA2, EPS, DECAY, MAX_NORM = 0.02, 0.9, 0.99, 1e-8, 0.01, 1.0


class Task:
    """Tokens whose successor is drawn from a fixed table, or (one in ten) from all of them."""

    def __init__(self, vocabulary: int, seed: int):
        gen = torch.Generator().manual_seed(seed)
        self.vocabulary = vocabulary
        self.successor = torch.randint(0, vocabulary, (vocabulary,), generator=gen)

    def batch(self, tokens: int, seed: int):
        gen = torch.Generator().manual_seed(seed)
        now = torch.randint(0, self.vocabulary, (tokens,), generator=gen)
        other = torch.randint(0, self.vocabulary, (tokens,), generator=gen)
        follows = torch.rand(tokens, generator=gen) < 0.9
        return now, torch.where(follows, self.successor[now], other)


def initial(vocabulary: int, width: int, seed: int) -> List[torch.Tensor]:
    """table, W, b in registration order."""
    gen = torch.Generator().manual_seed(seed + 1)
    return [torch.randn((vocabulary, width), generator=gen) * 0.02, torch.randn((vocabulary, width), generator=gen) * 0.02,
            torch.zeros(vocabulary)]


def run(replicas: int = 2, vocabulary: int = 512, width: int = 64, tokens: int = 1024, steps: int = 40, bits: int = 32,
        seed: int = 0, log=print) -> List[float]:
    """Trains and returns the mean loss over the replicas at every step."""
    device = harness.require_gpu()
    task, scale = Task(vocabulary, seed), math.sqrt(width)
    params = [p.to(device) for p in initial(vocabulary, width, seed)]
    numel = [p.numel() for p in params]
    n = len(numel)
    grads = harness.DeviceGrads(numel, [B.DDP_FP32] * n, replicas, fill=0)

    def grad(r: int, i: int) -> torch.Tensor:
        return grads.view(r, i).view(torch.float32).view(params[i].shape)

    losses = []
    with harness.Session(grads, 64 * 1024, B.DDP_PIPELINE_FUSED) as s:
        stream = s.backward_stream.cuda_stream
        emb = B.ddp_embedding_create(0, stream, vocabulary, width, tokens)
        opt = B.ddp_opt_create(0, stream)
        kind = B.DDP_STATE_8BIT if bits == 8 else B.DDP_STATE_FP32
        _, layout = B.ddp_opt_state_layout(numel, kind)
        state = torch.zeros(layout["bytes"], dtype=torch.uint8, device=device)       # step 0, moments of zero
        norm = torch.zeros(1, device=device)
        B.ddp_opt_register(opt, numel, [B.DDP_FP32] * n, [p.data_ptr() for p in params], [B.DDP_FP32] * n,
                           [grads.ptr(0, i) for i in range(n)])                      # the averages are replica 0's
        B.ddp_opt_set_groups(opt, None, [1.0, 1.0, 0.0])                             # the bias does not decay
        B.ddp_opt_set_state(opt, kind, state.data_ptr(), layout["bytes"])
        torch.cuda.synchronize()
        with torch.cuda.stream(s.backward_stream):
            table, weight, bias = params
            for step in range(steps):
                total = torch.zeros((), device=device)
                for r in range(replicas):
                    now, then = (x.to(device) for x in task.batch(tokens, (seed * 100003 + step) * 64 + r))
                    x = torch.empty((tokens, width), device=device)
                    B.ddp_embedding_lookup(emb, tokens, now.data_ptr(), 64, table.data_ptr(), B.DDP_FP32, width, scale,
                                           x.data_ptr(), B.DDP_FP32, width)
                    logp = torch.log_softmax(x @ weight.t() + bias, dim=1)
                    total += -logp.gather(1, then[:, None]).mean() / replicas
                    d = logp.exp()
                    d[torch.arange(tokens, device=device), then] -= 1.0
                    d /= tokens
                    grad(r, 2).copy_(d.sum(0))
                    grad(r, 1).copy_(d.t() @ x)
                    dx = d @ weight
                    g = grad(r, 0)
                    B.ddp_embedding_grad(emb, tokens, now.data_ptr(), 64, dx.data_ptr(), B.DDP_FP32, width, scale, -1, False,
                                         g.data_ptr(), B.DDP_FP32, width)
                for p in reversed(range(n)):                    # the table's gradient is the last to be ready
                    B.ddp_mark_ready(s.ctx, p)
                B.ddp_finalize_backward(s.ctx)
                B.ddp_opt_grad_norm(opt, 1.0, norm.data_ptr())
                B.ddp_opt_adamw_step(opt, LR, BETA1, BETA2, EPS, DECAY, 1.0, MAX_NORM, True)
                losses.append(total.item())
                if log and (step % 10 == 0 or step + 1 == steps):
                    log(f"step {step:3d}  loss {losses[-1]:.4f}  gradient norm {norm.item():.4f}", flush=True)
        torch.cuda.synchronize()
        B.ddp_opt_destroy(opt)
        B.ddp_embedding_destroy(emb)
    return losses


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--replicas", type=int, default=2)
    ap.add_argument("--vocabulary", type=int, default=512)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--tokens", type=int, default=1024, help="per replica and step")
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--bits", type=int, choices=(32, 8), default=32, help="of an element of the optimizer's state")
    a = ap.parse_args()
    losses = run(a.replicas, a.vocabulary, a.width, a.tokens, a.steps, a.bits)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")


if __name__ == "__main__":
    main()
