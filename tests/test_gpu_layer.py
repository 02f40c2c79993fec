"""The layer's pass, which calls lookup, norms, position bias, routing and all their gradients as a training step does, against the
same layer in plain 64-bit PyTorch on the CPU with autograd; and the training loop around it.

A gradient of the pass comes through at most some 25 products, norms and softmaxes one after the other, each of sums of up to 512 terms:
errors relative to the largest element stay below 25 * 512 u = 8e-4 (u = 2^-24), and the loss below that too.  The router's is a sum of
differences, s (1 - s) (g - mean of g) / (sum of the chosen s), whose two parts cancel (all of it where one expert is chosen: its weight is always 1):
an error of 8e-4 of each part is 8e-4 of the parts' magnitudes, and stays after they have cancelled."""
import dataclasses
import math

import pytest

pytestmark = pytest.mark.gpu


def plain(layer, s, p, balance, now, then, lengths, picked):
    """The loss, after its backward pass; `picked`: the experts that are to be chosen (compared with its own choice)."""
    import torch
    T, D, H, S, L = s.sequences * s.length, s.width, s.heads, s.sequences, s.length
    head = D // H
    flat = now.view(-1)
    x0 = torch.where(flat[:, None] >= 0, math.sqrt(D) * p["table"][flat.clamp(min=0)], 0.0)
    a = torch.nn.functional.layer_norm(x0, (D,), p["gamma1"], p["beta1"], layer.EPS)
    q, k, v = (a @ p["qkv"].t()).view(S, L, 3, H, head).permute(2, 0, 3, 1, 4)
    r = torch.arange(L)[None, :] - torch.arange(L)[:, None]
    t = (s.buckets - s.exact) * torch.log((-r).clamp(min=1).double() / s.exact) / math.log(s.distance / s.exact)
    far = (s.exact + (t + 1e-9).floor()).clamp(max=s.buckets - 1).long()
    bucket = torch.where(-r < s.exact, (-r).clamp(min=0), far)
    scores = q @ k.transpose(2, 3) / math.sqrt(head) + p["position"][bucket].permute(2, 0, 1)
    seen = (r <= 0)[None] & (torch.arange(L)[None, None, :] < lengths[:, None, None])
    scores = scores.masked_fill(~seen[:, None], -1e30)
    x1 = x0 + (torch.softmax(scores, 3) @ v).transpose(1, 2).reshape(T, D) @ p["out"].t()
    b = torch.nn.functional.layer_norm(x1, (D,), p["gamma2"], p["beta2"], layer.EPS)
    gate = torch.sigmoid(b @ p["router"].t())
    assert ((gate + balance).topk(s.chosen, dim=1).indices == picked).all()
    chosen = gate.gather(1, picked)
    w = chosen / chosen.sum(1, keepdim=True)
    w.retain_grad()
    mixed = torch.zeros_like(x1)
    for e in range(s.experts):
        t, n = (picked == e).nonzero(as_tuple=True)
        mixed = mixed.index_add(0, t, w[t, n][:, None] * (torch.relu(b[t] @ p[f"up{e}"].t()) @ p[f"down{e}"].t()))
    c = torch.nn.functional.layer_norm(x1 + mixed, (D,), p["gamma3"], p["beta3"], layer.EPS)
    real = flat >= 0
    loss = torch.nn.functional.cross_entropy((c @ p["vocabulary"].t())[real], then.view(-1)[real])
    loss.backward()
    parts = chosen * (1 - chosen) * (w.grad.abs() + (w.grad * w).abs().sum(1, keepdim=True)) / chosen.sum(1, keepdim=True)
    each = torch.zeros_like(gate).scatter_(1, picked, parts.detach())
    return loss, each.t() @ b.detach().abs()              # (the magnitudes of the router's gradient)


@pytest.mark.parametrize("sizes,seed", [({}, 0), (dict(vocabulary=91, width=60, heads=3, hidden=33, experts=13, chosen=3, sequences=5, length=37, buckets=11,
                                                       exact=4, distance=20), 1), (dict(experts=40, chosen=1, sequences=1, length=19), 2)])
def test_gradients(sizes, seed):
    import torch
    from paper_2006_15704_amd import layer, train
    s = dataclasses.replace(layer.Sizes(), **sizes)
    host = {k: v.double().requires_grad_() for k, v in layer.initial(s, seed).items()}
    gen = torch.Generator().manual_seed(seed)
    for k in "123":                                       # norms that do something
        for name in ("gamma" + k, "beta" + k):
            host[name] = (host[name].detach() + 0.2 * torch.randn(s.width, generator=gen)).float().double().requires_grad_()
    p = {k: v.detach().float().cuda() for k, v in host.items()}
    grad = {k: torch.full_like(v, 7.0) for k, v in p.items()}
    balance = 1e-2 * torch.randn(s.experts, generator=gen)
    now, then, lengths = train.sequences(train.Task(s.vocabulary, seed), s, seed)
    counts = torch.zeros(s.experts, dtype=torch.int32, device="cuda")
    model = layer.Layer(s, torch.cuda.current_stream().cuda_stream)
    seen = {}
    route = layer.B.ddp_router_route

    def watched(router, T, gate, *rest):                  # what the router chose, for the plain layer
        route(router, T, gate, *rest)
        seen["at"] = rest[3]
    layer.B.ddp_router_route = watched
    try:
        made = []
        empty = torch.empty

        def kept(*a, **k):
            made.append(empty(*a, **k))
            return made[-1]
        torch.empty = kept
        try:
            loss, load = model.step(p, grad, balance.cuda(), now.cuda(), then.cuda(), lengths.cuda(), counts)
        finally:
            torch.empty = empty
    finally:
        layer.B.ddp_router_route = route
    torch.cuda.synchronize()
    picked = next(t for t in made if t.data_ptr() == seen["at"]).long().cpu()
    model.close()
    assert load == torch.bincount(picked.view(-1), minlength=s.experts).tolist()
    want, parts = plain(layer, s, host, balance.double(), now, then, lengths, picked)
    assert abs(loss.item() - want.item()) <= 8e-4 * want.item()
    for k, v in host.items():
        if layer.expert_of(k) >= 0 and load[layer.expert_of(k)] == 0:
            assert (grad[k] == 7.0).all()
            continue
        got = grad[k].double().cpu()
        size = parts if k == "router" else v.grad.abs()
        assert (got - v.grad).abs().max() <= 8e-4 * size.max(), k


@pytest.mark.parametrize("bits,replicas,experts", [(32, 3, 8), (8, 2, 40)])
def test_the_loop_runs(bits, replicas, experts):
    """With 40 experts some are used by no replica, or by some alone."""
    from paper_2006_15704_amd import layer, train
    losses = train.run_layer(replicas, 3, bits, dataclasses.replace(layer.Sizes(), experts=experts, sequences=2, length=24), log=None)
    assert len(losses) == 3 and all(math.isfinite(x) for x in losses)
