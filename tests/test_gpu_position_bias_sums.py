"""Gradients of the position bias whose diagonals are long runs of equal scores over many sequences.

A lane adds a diagonal's scores in binary32 over at most 64 row groups of N (4 in binary32, 8 in 16 bits), one addition each (the first to 0), one more where
two lanes meet and three where four waves do, then in binary64; a block's sum is rounded to binary32, and so is the gradient.  Of equal scores c the
error is at most (64 N + 5) u of the result, u = 2^-24: 261 u = 1.6e-5 in binary32.  One chain over all sequences of a wave's share, 137000 additions here, is off by up to 1.6e-3."""
import numpy as np
import pytest

from layer_cases import BF16, FP16, FP32, U, close, lib, torch_type

pytestmark = pytest.mark.gpu


def constant(value, heads, batch, queries, keys, dt, kind, causal, both_lengths=None):
    """(gradient, what it is in 64 bits) of scores that are all the same; strides of 0: one row for all."""
    torch, d = lib()
    row = torch.full((keys,), value, dtype=torch_type(dt), device="cuda")
    grad = torch.zeros((kind[0], heads), device="cuda")
    lengths = None if both_lengths is None else torch.tensor(both_lengths, dtype=torch.int32, device="cuda")
    at = 0 if lengths is None else lengths.data_ptr()
    h = d.ddp_position_bias_create(0, 0, heads, *kind)
    first = d.ddp_position_bias_buckets(h)
    torch.cuda.synchronize()
    d.ddp_position_bias_grad(h, batch, queries, keys, 0, row.data_ptr(), dt, 0, 0, 0, 1.0, at, at, causal, False, grad.data_ptr(), FP32, heads)
    torch.cuda.synchronize()
    d.ddp_position_bias_destroy(h)
    want = np.zeros(kind[0])
    for q, k, times in [(queries, keys, batch)] if both_lengths is None else [(n, n, 1) for n in both_lengths]:
        r = np.arange(-(q - 1), 1 if causal else k)
        places = np.minimum(np.minimum(q, k - r) - np.maximum(0, -r), min(q, k))
        bucket = np.searchsorted(first, np.abs(r) if kind[3] else np.maximum(-r, 0), side="right") - 1 + (len(first) * (r > 0) if kind[3] else 0)
        want += times * np.bincount(bucket, weights=places, minlength=kind[0])
    return grad.double().cpu().numpy(), np.repeat(want[:, None] * float(row[0].double()), heads, axis=1)


@pytest.mark.parametrize("value", [0.1, 0.7, -0.0123])
@pytest.mark.parametrize("dt", [FP32, FP16, BF16])
def test_many_long_sequences(value, dt):
    """A block for each head and strip: a wave has a quarter of the row groups of all 134 sequences."""
    got, want = constant(value, 64, 134, 4096, 4096, dt, (32, 16, 128, False), False)
    n = 4 if dt == FP32 else 8
    close(got, want, (64 * n + 5) * U * np.abs(want), "gradient")


@pytest.mark.parametrize("heads,batch,queries,keys", [(1, 1, 4096, 4096), (3, 40, 1000, 1300), (64, 300, 520, 520), (16, 2000, 130, 64), (2, 5000, 1, 9)])
@pytest.mark.parametrize("dt", [FP32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_other_shapes(heads, batch, queries, keys, dt, causal):
    got, want = constant(0.7, heads, batch, queries, keys, dt, (64, 9, 300, True), causal)
    n = 4 if dt == FP32 else 8
    close(got, want, (64 * n + 5) * U * np.abs(want), "gradient")


def test_ragged_sequences():
    """Runs end in the middle of sequences, and some sequences have nothing."""
    lengths = [int(n) for n in np.random.default_rng(5).integers(0, 700, 400)]
    got, want = constant(0.1, 24, len(lengths), 699, 699, FP32, (64, 9, 300, True), False, lengths)
    close(got, want, 261 * U * np.abs(want), "gradient")
