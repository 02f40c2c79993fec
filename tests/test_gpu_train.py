"""The training loop that runs lookup, gradient, synchronization, norm and step together, against the same loop in plain
64-bit PyTorch on the CPU (autograd for the gradients, the step's formulas from the oracle)."""
import math

import numpy as np
import pytest

from oracle import operators as ops

pytestmark = pytest.mark.gpu


def plain(replicas, vocabulary, width, tokens, steps, seed):
    import torch
    from paper_2006_15704_amd import train
    task = train.Task(vocabulary, seed)
    params = [p.double().requires_grad_() for p in train.initial(vocabulary, width, seed)]
    state = [(np.zeros(p.numel()), np.zeros(p.numel())) for p in params]
    losses = []
    for step in range(steps):
        loss = 0.0
        for r in range(replicas):
            now, then = task.batch(tokens, (seed * 100003 + step) * 64 + r)
            x = math.sqrt(width) * params[0][now]
            loss = loss + torch.nn.functional.cross_entropy(x @ params[1].t() + params[2], then) / replicas
        grads = [g.numpy().reshape(-1) for g in torch.autograd.grad(loss, params)]
        losses.append(loss.item())
        norm = ops.grad_norm(grads)
        for i, p in enumerate(params):
            new, m, v = ops.adamw(p.detach().numpy().reshape(-1), grads[i], *state[i], step + 1, train.LR, train.BETA1, train.BETA2,
                                  train.EPS, train.DECAY * (i < 2), 1.0, train.MAX_NORM, norm)
            state[i] = (m, v)
            params[i] = torch.from_numpy(new).view(p.shape).requires_grad_()
    return losses


@pytest.mark.parametrize("bits", [32, 8])
def test_training_follows_the_plain_loop(bits):
    """32 bits: the losses agree closely for as long as roundings have not grown (a step divides by the root of a moment
    that starts at 0: gradients near 0 get updates of a rounding error's sign, but move the loss little).
    8 bits: the first step's updates do not see the codes yet; later ones follow within a few per cent."""
    from paper_2006_15704_amd import train
    sizes = dict(replicas=3, vocabulary=96, width=32, tokens=256, steps=12, seed=5)
    want = plain(**sizes)
    got = train.run(bits=bits, log=None, **sizes)
    assert abs(got[0] - want[0]) <= 1e-4 * want[0] and abs(got[1] - want[1]) <= 1e-3 * want[1]
    for a, b in zip(got, want):
        assert abs(a - b) <= (2e-3 if bits == 32 else 5e-2) * b
    assert got[-1] < 0.8 * got[0]


@pytest.mark.parametrize("bits", [32, 8])
def test_training_learns(bits):
    from paper_2006_15704_amd import train
    losses = train.run(steps=60, bits=bits, log=None)
    assert losses[-1] < 0.5 * losses[0]
