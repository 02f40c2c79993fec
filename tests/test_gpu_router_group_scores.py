"""Scores of groups whose two largest keys, or their sum, leave binary32: the opened groups are those of binary64.

Tolerances are those of the routing tests: choices are equal, weights are off by their R u."""
import numpy as np
import pytest

from test_gpu_router import SIGMOID, SOFTMAX, check_route

pytestmark = pytest.mark.gpu

KINDS = [(8, 2, 4, 1, 2), (8, 3, 4, 2, 2), (64, 6, 4, 2, 2), (160, 6, 8, 3, 2), (256, 8, 8, 4, 2), (33, 3, 11, 2, 2), (40, 4, 8, 2, 1)]


def check(kind, score, times, logits, bias):
    check_route(len(logits), kind, score, True, logits=logits, bias=bias.astype(np.float32), times=times)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("times", [1, 1000])
def test_sums_below_binary32(kind, score, times):
    """Whole groups at biases between half the lowest value and the lowest, the later ones higher; then behind a group without any
    expert.  Within a group the keys are far apart."""
    E, groups = kind[0], kind[2]
    logits = np.random.default_rng(E).standard_normal((24, E))
    apart = 2e35 * np.tile(np.arange(E // groups), groups)
    check(kind, score, times, logits, np.repeat(np.linspace(-3.3e38, -1.8e38, groups), E // groups) + apart)
    logits[::2, :E // groups] = -np.inf
    check(kind, score, times, logits, apart - 2.5e38)
    check(kind, score, times, logits, np.full(E, -2.5e38))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("times", [1, 1000])
def test_sums_above_binary32(kind, score, times):
    """The first group has the largest key and the lowest, whose sum is 0; the others have two whose sum, or either with the largest
    bias added, is beyond binary32."""
    E, groups = kind[0], kind[2]
    each = E // groups
    logits = np.random.default_rng(E).standard_normal((24, E))
    for most in (1.3e38, 1.6e38):
        bias = np.repeat(np.linspace(1.1e38, most, groups), each) + 2e35 * np.tile(np.arange(each), groups)
        bias[:each] = -2e38
        bias[0] = 2e38
        check(kind, score, times, logits, bias)
