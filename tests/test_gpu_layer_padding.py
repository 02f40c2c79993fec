"""Tokens behind a sequence's end in the layer's pass, and what the training loop makes of the experts' counts.

Gradients of a pass are off by at most 8e-4 of their largest element (test_gpu_layer.py), of two passes of the same tokens by twice that."""
import dataclasses

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def one_pass(s, seed, now, then, lengths):
    """(loss, rows of every expert, counts, gradients) of a step; gradients hold 7 before it."""
    import torch
    from paper_2006_15704_amd import layer
    p = {k: v.cuda() for k, v in layer.initial(s, seed).items()}
    grad = {k: torch.full_like(v, 7.0) for k, v in p.items()}
    counts = torch.full((s.experts,), 99, dtype=torch.int32, device="cuda")
    model = layer.Layer(s, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    loss, rows = model.step(p, grad, torch.zeros(s.experts, device="cuda"), now.cuda(), then.cuda(), lengths.cuda(), counts)
    torch.cuda.synchronize()
    model.close()
    return loss.item(), rows, counts.tolist(), {k: v.cpu() for k, v in grad.items()}


@pytest.mark.parametrize("sizes,seed", [(dict(experts=40, sequences=2, length=24), 1), (dict(experts=40, chosen=1, sequences=1, length=19), 7),
                                        (dict(experts=40, chosen=3, sequences=2, length=30), 8)])
def test_padding_counts_for_nothing(sizes, seed):
    """The same sequences with more padding: the same counts, and the same gradients.  In each case there are experts that
    padding alone would have chosen: they count no token and have no gradient."""
    import torch
    from paper_2006_15704_amd import layer, train
    s = dataclasses.replace(layer.Sizes(), **sizes)
    now, then, lengths = train.sequences(train.Task(s.vocabulary, seed), s, seed)
    more = [torch.nn.functional.pad(x, (0, 13), value=-1) for x in (now, then.clamp(min=0))]
    loss, rows, counts, grad = one_pass(s, seed, now, then, lengths)
    loss2, _, counts2, grad2 = one_pass(dataclasses.replace(s, length=s.length + 13), seed, *more, lengths)
    assert sum(counts) == s.chosen * int(lengths.sum()) == sum(counts2)
    assert counts == counts2
    alone = [e for e in range(s.experts) if rows[e] > 0 and counts[e] == 0]
    assert alone, "no expert that padding alone has chosen"
    assert abs(loss - loss2) <= 2 * 8e-4 * loss
    for k, v in grad.items():
        e = layer.expert_of(k)
        if e >= 0 and counts[e] == 0:
            assert ((v == 0.0) | (v == 7.0)).all() and (v == v.view(-1)[0]).all()
        else:
            assert (v - grad2[k]).abs().max() <= 2 * 8e-4 * v.abs().max(), k


@pytest.mark.parametrize("bits,replicas,sizes", [(32, 2, dict(experts=40, sequences=1, length=12)), (8, 3, dict(experts=32, chosen=1, sequences=1, length=16)),
                                                 (32, 1, dict(experts=8, sequences=2, length=24))])
def test_what_the_loop_does_with_counts(bits, replicas, sizes, monkeypatch):
    """Participation is a count above 0, parameters of experts that no replica used keep their bits and the others do not, and the balance
    bias moves by the rate towards the mean of the counts."""
    import torch
    from oracle import layer as ops
    from paper_2006_15704_amd import layer, train
    s = dataclasses.replace(layer.Sizes(), **sizes)
    names = layer.names(s)
    tokens, flags, before, after, moves = [], {}, [], [], []

    step, mark, balance = layer.Layer.step, train.B.ddp_mark_ready_local, train.B.ddp_router_balance
    held = {}

    def watched_step(self, p, grad, bias, now, then, lengths, counts):
        if len(tokens) % replicas == 0:
            held.update(p=p, bias=bias)
            before.append({k: v.clone() for k, v in p.items()})
        out = step(self, p, grad, bias, now, then, lengths, counts)
        tokens.append((int((now >= 0).sum()), counts.tolist()))
        return out

    def watched_mark(ctx, i, used):
        flags.setdefault(len(before) - 1, {})[i] = [bool(u) for u in used]
        return mark(ctx, i, used)

    def watched_balance(router, n, counts, rate, bias, bias_out):
        after.append({k: v.clone() for k, v in held["p"].items()})
        old = held["bias"].clone()
        balance(router, n, counts, rate, bias, bias_out)
        moves.append((rate, old, held["bias"].clone()))

    monkeypatch.setattr(layer.Layer, "step", watched_step)
    monkeypatch.setattr(train.B, "ddp_mark_ready_local", watched_mark)
    monkeypatch.setattr(train.B, "ddp_router_balance", watched_balance)
    steps = 3
    losses = train.run_layer(replicas, steps, bits, s, log=None)
    torch.cuda.synchronize()
    assert len(losses) == len(before) == len(after) == steps and len(tokens) == steps * replicas
    unused = used = 0
    for n in range(steps):
        load = [c for _, c in tokens[n * replicas:(n + 1) * replicas]]
        for many, c in tokens[n * replicas:(n + 1) * replicas]:
            assert sum(c) == s.chosen * many
        for i, k in enumerate(names):
            e = layer.expert_of(k)
            old, new = before[n][k], after[n][k]
            if e < 0:
                assert i not in flags[n]
                continue
            assert flags[n][i] == [c[e] > 0 for c in load], (n, k)
            if any(c[e] for c in load):
                used += 1
                assert not torch.equal(old, new), (n, k)
            else:
                unused += 1
                assert torch.equal(old, new), (n, k)
        rate, old, new = moves[n]
        assert rate == train.BALANCE
        want = ops.balance(np.array(load), old.cpu().numpy(), rate)
        assert torch.equal(new.cpu(), torch.from_numpy(want))
        assert not torch.equal(old, new)
    assert used and (unused or s.experts == 8)
