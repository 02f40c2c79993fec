"""The oracle of the operators inside a layer: gradients against differences of the forward formulas, buckets and
choices against small cases written out by hand."""
import math

import numpy as np
import pytest

from oracle import layer as ops


def differences(f, x, step=1e-5):
    out = np.zeros(x.size)
    for i in range(x.size):
        up, down = x.copy().reshape(-1), x.copy().reshape(-1)
        up[i] += step
        down[i] -= step
        out[i] = (f(up.reshape(x.shape)) - f(down.reshape(x.shape))) / (2 * step)
    return out.reshape(x.shape)


def test_norm_of_a_known_row():
    y, mean, rstd = ops.norm(np.array([[1.0, 3.0]]), np.array([2.0, 2.0]), np.array([0.5, 0.5]), 0.0)
    assert mean[0] == 2.0 and rstd[0] == 1.0 and y.tolist() == [[-1.5, 2.5]]


def test_norm_gradients_are_those_of_differences():
    rng = np.random.default_rng(0)
    s, gamma, beta, dy = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    eps = 1e-3

    def loss(s=s, gamma=gamma, beta=beta):
        return float((ops.norm(s, gamma, beta, eps)[0] * dy).sum())

    _, mean, rstd = ops.norm(s, gamma, beta, eps)
    dx, dgamma, dbeta = ops.norm_grad(dy, s, mean, rstd, gamma)
    np.testing.assert_allclose(dx, differences(lambda v: loss(s=v), s), atol=1e-8)
    np.testing.assert_allclose(dgamma, differences(lambda v: loss(gamma=v), gamma), atol=1e-8)
    np.testing.assert_allclose(dbeta, differences(lambda v: loss(beta=v), beta), atol=1e-8)


def test_buckets_of_known_distances():
    # 8 buckets of one direction, 4 of them exact, 4 steps from 4 to 64: a factor of 2 each
    of = [ops.bucket(-d, 8, 4, 64, False) for d in range(70)]
    assert of[:4] == [0, 1, 2, 3]
    assert [of.index(k) for k in range(4, 8)] == [4, 8, 16, 32]
    assert of[64] == of[69] == 7
    assert ops.bucket(5, 8, 4, 64, False) == 0
    # both directions: keys behind the query come after the others
    assert [ops.bucket(r, 8, 4, 64, True) for r in (0, -1, 1, -3, 3, -9, 9)] == [0, 1, 5, 3, 7, 3, 7]


@pytest.mark.parametrize("buckets,exact,distance", [(32, 16, 128), (32, 8, 128), (7, 1, 9), (20, 3, 700)])
def test_buckets_follow_the_logarithm(buckets, exact, distance):
    for d in range(1, 3 * distance):
        k = ops.bucket(-d, buckets, exact, distance, False)
        if d < exact:
            assert k == d
            continue
        t = (buckets - exact) * math.log(d / exact) / math.log(distance / exact)
        if abs(t - round(t)) > 1e-9:
            assert k == min(buckets - 1, exact + math.floor(t))
        else:
            assert k == min(buckets - 1, exact + round(t))


def test_bias_gradient_is_that_of_differences():
    rng = np.random.default_rng(1)
    B, H, Q, K, buckets = 2, 3, 4, 6, (6, 2, 5, True)
    table, ds = rng.standard_normal((6, H)), rng.standard_normal((B, H, Q, K))
    seen = ops.visible(B, Q, K, 1, True, [6, 3], [4, 2])
    places = ops.bucket_places(Q, K, 1, *buckets)

    def loss(table):
        return float(sum((np.where(seen[b], table[places, h], 0.0) * ds[b, h]).sum() for b in range(B) for h in range(H)))

    grad, magnitude = ops.bias_grad(ds, seen, places, 6)
    np.testing.assert_allclose(grad, differences(loss, table), atol=1e-8)
    assert (magnitude >= np.abs(grad) - 1e-12).all()


def test_choices_of_a_known_token():
    x = np.array([[1.0, 3.0, 3.0, 2.0]])
    zero = np.zeros(4)
    experts, weights = ops.route(x, zero, 3, 1, 1, 1, ops.SIGMOID, True, 2.0)
    assert experts.tolist() == [[1, 2, 3]] and abs(weights.sum() - 2.0) < 1e-12
    # a bias chooses, and is no part of the weights
    experts, weights = ops.route(x, np.array([9.0, 0, 0, 0]), 1, 1, 1, 1, ops.SIGMOID, False, 1.0)
    assert experts.tolist() == [[0]] and abs(weights[0, 0] - 1 / (1 + math.exp(-1.0))) < 1e-15
    # two groups: {0, 1} has the larger sum, {2, 3} the larger key
    x = np.array([[2.0, 2.0, 3.0, -9.0]])
    assert ops.route(x, zero, 1, 2, 1, 2, ops.SIGMOID, True, 1.0)[0].tolist() == [[0]]
    assert ops.route(x, zero, 1, 2, 1, 1, ops.SIGMOID, True, 1.0)[0].tolist() == [[2]]
    # masked experts leave places over
    x = np.array([[-np.inf, 1.0, np.nan, -np.inf], [-np.inf] * 4])
    experts, weights = ops.route(x, zero, 2, 1, 1, 1, ops.SIGMOID, True, 1.0)
    assert experts.tolist() == [[1, -1], [-1, -1]] and weights.tolist() == [[1.0, 0.0], [0.0, 0.0]]
    assert ops.route(x, zero, 2, 1, 1, 1, ops.SOFTMAX, True, 1.0)[0].tolist() == [[-1, -1], [-1, -1]]


@pytest.mark.parametrize("score", [ops.SOFTMAX, ops.SIGMOID])
@pytest.mark.parametrize("renormalise", [False, True])
def test_routing_gradient_is_that_of_differences(score, renormalise):
    rng = np.random.default_rng(2)
    x, dw = rng.standard_normal((3, 8)), rng.standard_normal((3, 3))
    experts, _ = ops.route(x, np.zeros(8), 3, 1, 1, 1, score, renormalise, 1.5)

    def loss(x):
        s = ops.scores(x, score)
        w = np.take_along_axis(s, experts, 1)
        return float((1.5 * (w / w.sum(axis=1, keepdims=True) if renormalise else w) * dw).sum())

    dx, _ = ops.route_grad(x, experts, dw, score, renormalise, 1.5)
    np.testing.assert_allclose(dx, differences(loss, x), atol=1e-8)


def test_balance_moves_towards_the_mean():
    counts = np.array([[1, 5, 3, 3], [2, 4, 3, 3]])
    assert ops.balance(counts, np.zeros(4, dtype=np.float32), 0.5).tolist() == [0.5, -0.5, 0.0, 0.0]
