"""One transformer layer between an embedding and a vocabulary, in binary32, its passes written out: causal attention
with a learned relative position bias, and experts that a router chooses, each behind a layer norm.

    x0 = scale * table[token]           a = norm(x0)              x1 = x0 + attention(a)
    b = norm(x1)                        x2 = x1 + experts(b)      logits = norm(x2) W^T

The library does what is not a matrix product: lookup, norms with their residual sums, position bias, routing, and the
gradients of all of them, which go straight into the gradient tensors that a synchronization averages.  The products, the attention's
softmax and the loss are PyTorch's.
"""
from __future__ import annotations

import math
from dataclasses import dataclass
from typing import Dict, List, Sequence, Tuple

import torch

from . import binding as B

EPS = 1e-5


@dataclass
class Sizes:
    vocabulary: int = 256
    width: int = 64
    heads: int = 4
    hidden: int = 64          # of an expert
    experts: int = 8
    chosen: int = 2
    sequences: int = 8
    length: int = 64
    buckets: int = 16
    exact: int = 8
    distance: int = 48


def names(s: Sizes) -> List[str]:
    """Parameters in registration order."""
    out = ["table", "position", "gamma1", "beta1", "qkv", "out", "gamma2", "beta2", "router"]
    for e in range(s.experts):
        out += [f"up{e}", f"down{e}"]
    return out + ["gamma3", "beta3", "vocabulary"]


def expert_of(name: str) -> int:
    """The expert that a parameter belongs to, or -1."""
    for kind in ("up", "down"):
        if name.startswith(kind) and name[len(kind):].isdigit():
            return int(name[len(kind):])
    return -1


def initial(s: Sizes, seed: int) -> Dict[str, torch.Tensor]:
    gen = torch.Generator().manual_seed(seed + 1)
    D = s.width

    def weight(*shape):
        return torch.randn(shape, generator=gen) / math.sqrt(shape[-1])

    p = {"table": torch.randn((s.vocabulary, D), generator=gen) / math.sqrt(D),
         "position": torch.randn((s.buckets, s.heads), generator=gen) * 0.2, "qkv": weight(3 * D, D), "out": weight(D, D),
         "router": weight(s.experts, D), "vocabulary": weight(s.vocabulary, D)}
    for e in range(s.experts):
        p[f"up{e}"], p[f"down{e}"] = weight(s.hidden, D), weight(D, s.hidden)
    for k in "123":
        p["gamma" + k], p["beta" + k] = torch.ones(D), torch.zeros(D)
    return {n: p[n] for n in names(s)}


class Layer:
    """The handles of a layer on one stream, and its passes."""

    def __init__(self, sizes: Sizes, stream: int):
        s = self.sizes = sizes
        self.tokens = s.sequences * s.length
        self.embedding = B.ddp_embedding_create(0, stream, s.vocabulary, s.width, self.tokens)
        self.norm = B.ddp_layernorm_create(0, stream, s.width)
        self.position = B.ddp_position_bias_create(0, stream, s.heads, s.buckets, s.exact, s.distance, False)
        self.router = B.ddp_router_create(0, stream, s.experts, s.chosen, score=B.DDP_SCORE_SIGMOID)

    def close(self) -> None:
        B.ddp_router_destroy(self.router)
        B.ddp_position_bias_destroy(self.position)
        B.ddp_layernorm_destroy(self.norm)
        B.ddp_embedding_destroy(self.embedding)

    def _norm(self, x, residual, gamma, beta):
        """(norm of x + residual, the sum, its statistics)."""
        T, D = x.shape
        y, mean, rstd = torch.empty_like(x), torch.empty(T, device=x.device), torch.empty(T, device=x.device)
        total = x if residual is None else torch.empty_like(x)
        B.ddp_layernorm_forward(self.norm, T, x.data_ptr(), B.DDP_FP32, D, 0 if residual is None else residual.data_ptr(), D, gamma.data_ptr(),
                                beta.data_ptr(), B.DDP_FP32, EPS, 0 if residual is None else total.data_ptr(), D, y.data_ptr(), B.DDP_FP32, D,
                                mean.data_ptr(), rstd.data_ptr())
        return y, total, (mean, rstd)

    def _norm_grad(self, dy, total, stats, gamma, along, dgamma, dbeta):
        """The gradient of the sum; `along`: what flows back along it by itself."""
        T, D = dy.shape
        dx = torch.empty_like(dy)
        B.ddp_layernorm_backward(self.norm, T, dy.data_ptr(), B.DDP_FP32, D, total.data_ptr(), B.DDP_FP32, D, stats[0].data_ptr(),
                                 stats[1].data_ptr(), gamma.data_ptr(), B.DDP_FP32, 0 if along is None else along.data_ptr(), D, dx.data_ptr(),
                                 D, False, dgamma.data_ptr(), dbeta.data_ptr(), B.DDP_FP32)
        return dx

    def step(self, p: Dict[str, torch.Tensor], grad: Dict[str, torch.Tensor], balance: torch.Tensor, now: torch.Tensor, then: torch.Tensor,
             lengths: torch.Tensor, counts: torch.Tensor) -> Tuple[torch.Tensor, Sequence[int]]:
        """One replica's forward and backward pass: writes its gradients and counts (int32 [experts]: the tokens of each expert).
        now, then: int64 [sequences, length]; lengths: int32 [sequences], behind which tokens are -1.  Returns (mean loss, the rows that the
        router gave each expert, those behind a sequence's end among them).  Gradients of experts without a row are left as they are; where all
        their rows are behind an end they are zeros, and their count is 0."""
        s, T, D, H = self.sizes, self.tokens, self.sizes.width, self.sizes.heads
        S, L, scale = s.sequences, s.length, math.sqrt(s.width)
        head = D // H
        x0 = torch.empty((T, D), device=now.device)
        B.ddp_embedding_lookup(self.embedding, T, now.data_ptr(), 64, p["table"].data_ptr(), B.DDP_FP32, D, scale, x0.data_ptr(), B.DDP_FP32, D)
        a, _, stats1 = self._norm(x0, None, p["gamma1"], p["beta1"])
        qkv = (a @ p["qkv"].t()).view(S, L, 3, H, head).permute(2, 0, 3, 1, 4).contiguous()
        q, k, v = qkv[0] / math.sqrt(head), qkv[1], qkv[2]
        scores = q @ k.transpose(2, 3).contiguous()
        B.ddp_position_bias_apply(self.position, S, L, L, 0, p["position"].data_ptr(), B.DDP_FP32, H, 1.0, lengths.data_ptr(), True, -1e30, True,
                                  scores.data_ptr(), B.DDP_FP32, *scores.stride()[:3])
        prob = torch.softmax(scores, dim=3)
        context = (prob @ v).transpose(1, 2).reshape(T, D)
        b, x1, stats2 = self._norm(context @ p["out"].t(), x0, p["gamma2"], p["beta2"])
        gate = b @ p["router"].t()
        chosen = torch.empty((T, s.chosen), dtype=torch.int32, device=now.device)
        weights = torch.empty((T, s.chosen), device=now.device)
        rows = torch.empty(s.experts, dtype=torch.int32, device=now.device)
        B.ddp_router_route(self.router, T, gate.data_ptr(), B.DDP_FP32, s.experts, balance.data_ptr(), chosen.data_ptr(), weights.data_ptr(),
                           B.DDP_FP32, rows.data_ptr())
        # rows behind a sequence's end are routed with the rest, and that is all: no expert has them, no count and no gradient
        picked = chosen.masked_fill((now.view(-1) < 0)[:, None], -1)
        counts.copy_((picked.view(-1, 1) == torch.arange(s.experts, device=now.device)).sum(0))
        mixed, kept = torch.zeros((T, D), device=now.device), {}
        load = rows.tolist()
        for e in range(s.experts):
            if load[e] == 0:
                continue
            t, n = (picked == e).nonzero(as_tuple=True)
            up = b[t] @ p[f"up{e}"].t()
            down = torch.relu(up) @ p[f"down{e}"].t()
            mixed.index_add_(0, t, weights[t, n][:, None] * down)
            kept[e] = t, n, up, down
        c, x2, stats3 = self._norm(mixed, x1, p["gamma3"], p["beta3"])
        logp = torch.log_softmax(c @ p["vocabulary"].t(), dim=1)
        real = (now.view(-1) >= 0).nonzero().view(-1)
        follow = then.view(-1)[real]
        loss = -logp[real, follow].mean()
        # backward
        d = torch.zeros_like(logp)
        d[real] = logp[real].exp()
        d[real, follow] -= 1.0
        d /= len(real)
        grad["vocabulary"].copy_(d.t() @ c)
        dx2 = self._norm_grad(d @ p["vocabulary"], x2, stats3, p["gamma3"], None, grad["gamma3"], grad["beta3"])
        db, dweights = torch.zeros_like(b), torch.zeros_like(weights)
        for e, (t, n, up, down) in kept.items():
            dweights[t, n] = (dx2[t] * down).sum(1)
            ddown = weights[t, n][:, None] * dx2[t]
            grad[f"down{e}"].copy_(ddown.t() @ torch.relu(up))
            dup = (ddown @ p[f"down{e}"]) * (up > 0)
            grad[f"up{e}"].copy_(dup.t() @ b[t])
            db.index_add_(0, t, dup @ p[f"up{e}"])
        dgate = torch.empty_like(gate)
        B.ddp_router_grad(self.router, T, gate.data_ptr(), B.DDP_FP32, s.experts, picked.data_ptr(), dweights.data_ptr(), B.DDP_FP32, dgate.data_ptr(),
                          s.experts)
        grad["router"].copy_(dgate.t() @ b)
        db += dgate @ p["router"]
        dx1 = self._norm_grad(db, x1, stats2, p["gamma2"], dx2, grad["gamma2"], grad["beta2"])
        grad["out"].copy_(dx1.t() @ context)
        dcontext = (dx1 @ p["out"]).view(S, L, H, head).transpose(1, 2).contiguous()
        dprob = dcontext @ v.transpose(2, 3).contiguous()
        ds = prob * (dprob - (dprob * prob).sum(3, keepdim=True))
        B.ddp_position_bias_grad(self.position, S, L, L, 0, ds.data_ptr(), B.DDP_FP32, *ds.stride()[:3], 1.0, lengths.data_ptr(), lengths.data_ptr(),
                                 True, False, grad["position"].data_ptr(), B.DDP_FP32, H)
        dqkv = torch.stack([ds @ k / math.sqrt(head), ds.transpose(2, 3).contiguous() @ q, prob.transpose(2, 3).contiguous() @ dcontext])
        dqkv = dqkv.permute(1, 3, 0, 2, 4).reshape(T, 3 * D)
        grad["qkv"].copy_(dqkv.t() @ a)
        dx0 = self._norm_grad(dqkv @ p["qkv"], x0, stats1, p["gamma1"], dx1, grad["gamma1"], grad["beta1"])
        B.ddp_embedding_grad(self.embedding, T, now.data_ptr(), 64, dx0.data_ptr(), B.DDP_FP32, D, scale, -1, False, grad["table"].data_ptr(),
                             B.DDP_FP32, D)
        return loss, load
