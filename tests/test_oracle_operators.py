"""Pins of the operators' oracle: hand-worked values, gradients against
differences, and what the 8-bit codes promise."""
import numpy as np
import pytest

from oracle import operators as ops


def test_lookup_by_hand():
    table = np.arange(6, dtype=np.float32).reshape(3, 2)
    out = ops.lookup(table, np.array([2, -1, 0, 3]), 0.5)
    assert out.tolist() == [[2.0, 2.5], [0.0, 0.0], [0.0, 0.5], [0.0, 0.0]]


@pytest.mark.parametrize("padding", [-1, 1])
def test_embedding_grad_against_differences(padding):
    """d/d table of sum(w * lookup(table)), by central differences (the map is linear, so they are exact up to
    rounding: 2e-16 * |values| / step)."""
    rng = np.random.default_rng(3)
    rows, width, tokens, scale = 5, 3, 11, 1.7
    ids = rng.integers(-1, rows + 1, size=tokens)
    w = rng.standard_normal((tokens, width))
    w_used = np.where((ids == padding)[:, None], 0.0, w)      # a padding token's row is not learned from
    table = rng.standard_normal((rows, width))
    grad, _ = ops.embedding_grad(rows, ids, w, scale, padding)
    h = 0.5
    for r in range(rows):
        for c in range(width):
            up, down = table.copy(), table.copy()
            up[r, c] += h
            down[r, c] -= h
            d = ((ops.lookup(up, ids, scale) - ops.lookup(down, ids, scale)) * w_used).sum() / (2 * h)
            assert abs(d - grad[r, c]) < 1e-12


def test_embedding_grad_adds():
    grad, _ = ops.embedding_grad(3, np.array([1, 1, 7]), np.ones((3, 2)), 2.0, -1, np.full((3, 2), 10.0))
    assert grad.tolist() == [[10.0, 10.0], [14.0, 14.0], [10.0, 10.0]]


def test_first_adamw_step_by_hand():
    """From zero moments the first step moves every element by lr against its gradient's sign."""
    p = np.array([1.0, -2.0, 0.5])
    g = np.array([0.25, -4.0, 0.0])
    new, m, v = ops.adamw(p, g, np.zeros(3), np.zeros(3), 1, 0.1, 0.9, 0.99, 0.0 + 1e-30, 0.5)
    np.testing.assert_allclose(m, [0.025, -0.4, 0.0])
    np.testing.assert_allclose(v, [0.000625, 0.16, 0.0])
    np.testing.assert_allclose(new, [1.0 - 0.05 - 0.1, -2.0 + 0.1 + 0.1, 0.5 - 0.025])


def test_clip_scales_to_the_norm():
    g = np.array([3.0, 4.0])
    _, m, _ = ops.adamw(g, g, np.zeros(2), np.zeros(2), 1, 0.1, 0.0, 0.9, 1e-8, 0.0, 1.0, 1.0, ops.grad_norm([g]))
    np.testing.assert_allclose(m, [0.6, 0.8], rtol=1e-6)
    _, m, _ = ops.adamw(g, g, np.zeros(2), np.zeros(2), 1, 0.1, 0.0, 0.9, 1e-8, 0.0, 1.0, 50.0, ops.grad_norm([g]))
    np.testing.assert_allclose(m, g)


def test_codes():
    """Every code is the nearest code of what it stands for, the top is held exactly, nothing positive becomes 0."""
    k = np.arange(-127, 128)
    k = np.concatenate([k, [0]])
    held = ops.held_first(k, np.array([3.0]))
    codes, tops, _ = ops.nearest_first(held)
    assert tops[0] == 3.0 and (codes == k).all()
    k = np.arange(256)
    held = ops.held_second(k, np.array([5.0]))
    codes, tops, _ = ops.nearest_second(held)
    assert tops[0] == 5.0 and (codes == k).all()
    v = np.array([1.0, 1e-30, 0.0])
    codes, _, _ = ops.nearest_second(v)
    assert codes.tolist() == [255.0, 1.0, 0.0]
    # half a step at the top: 0.8 % of the first moment, of the second
    x = np.linspace(0.5, 1.0, 999)
    codes, tops, _ = ops.nearest_first(x)
    assert np.abs(ops.held_first(codes, tops) / x - 1).max() < 0.0115
    codes, tops, _ = ops.nearest_second(x)
    assert np.abs(ops.held_second(codes, tops) / x - 1).max() < 0.0095


def test_clipping_by_norms_that_are_not_finite():
    """min(1, NaN) is NaN; an infinite norm leaves nothing of a finite gradient."""
    p, g, m, v = np.ones(3), np.array([0.5, -1.0, 2.0]), np.full(3, 0.1), np.full(3, 0.2)
    for norm, factor in ((np.inf, 0.0), (np.nan, np.nan), (10.0, 1.0 / (10.0 + 1e-6)), (0.5, 1.0)):
        got = ops.adamw(p, g, m, v, 3, 1e-2, 0.9, 0.99, 1e-8, 0.1, 1.0, 1.0, norm)
        want = ops.adamw(p, g * factor, m, v, 3, 1e-2, 0.9, 0.99, 1e-8, 0.1)
        for x, y in zip(got, want):
            np.testing.assert_allclose(x, y, rtol=1e-15, equal_nan=True)
