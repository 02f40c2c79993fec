"""Renormalised weights with a large scale: scale / (sum of the chosen scores) leaves binary32 where the weights do not."""
import numpy as np
import pytest

from test_gpu_router import FP32, SIGMOID, SOFTMAX, KINDS, check_route

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scale", [1e12, 3e38, 1e-30])
@pytest.mark.parametrize("times", [1, 1000])
def test_small_sums(kind, scale, times):
    """Sigmoids of logits near -64, and softmaxes of which the bias chooses experts that are 60 below the largest."""
    E = kind[0]
    rng = np.random.default_rng(E)
    logits = rng.standard_normal((24, E)) - 64.0
    check_route(24, kind, SIGMOID, True, scale=scale, logits=logits, bias=False, times=times)
    logits[:, ::2] += 60.0
    bias = np.zeros(E, dtype=np.float32)
    bias[1::2] = 8.0 + rng.integers(0, 40, E // 2) * 0.125
    check_route(24, kind, SOFTMAX, True, FP32, scale=scale, logits=logits, bias=bias, times=times)
