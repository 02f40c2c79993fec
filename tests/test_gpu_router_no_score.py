"""The gradient of sigmoids that are 0 in binary64: 1 / (1 + exp(-x)) for x below -709.78, where exp(-x) is beyond it.  Their weights are 0
whatever the logits are, and so is their gradient."""
import numpy as np
import pytest

from test_gpu_router import BF16, FP32, SIGMOID, check_grad, check_route, lib

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [(4, 2, 1, 1, 1), (64, 2, 1, 1, 1), (256, 8, 8, 4, 2), (60, 4, 1, 1, 1), (512, 16, 1, 1, 1)])
@pytest.mark.parametrize("lowest,highest", [(-744.0, -711.0), (-2000.0, -746.0), (-700.0, -600.0)])
def test_weights_and_gradient(kind, lowest, highest):
    rng = np.random.default_rng(kind[0])
    logits = rng.uniform(lowest, highest, (40, kind[0]))
    check_route(40, kind, SIGMOID, True, logits=logits, bias=False)
    check_grad(40, kind, SIGMOID, True, logits=logits)
    check_grad(40, kind, SIGMOID, True, BF16, logits=logits)


def test_the_border():
    """The last number of binary32 whose sigmoid is above 0 has weights, the next has none; so have the gradients."""
    torch, d = lib()
    last = np.float32(-709.78265)
    assert 1.0 / (1.0 + np.exp(-np.float64(last))) > 0.0
    below = np.nextafter(last, np.float32(-1e3))
    with np.errstate(over="ignore"):
        assert 1.0 / (1.0 + np.exp(-np.float64(below))) == 0.0
    x = torch.tensor([[last, last], [last, below], [below, below]], device="cuda")
    experts, weights = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.zeros((3, 2), device="cuda")
    dw, dx = torch.tensor([[1.0, -1.0]] * 3, device="cuda"), torch.full((3, 2), 9.0, device="cuda")
    h = d.ddp_router_create(0, 0, 2, 2, score=SIGMOID)
    torch.cuda.synchronize()
    d.ddp_router_route(h, 3, x.data_ptr(), FP32, 2, 0, experts.data_ptr(), weights.data_ptr(), FP32)
    d.ddp_router_grad(h, 3, x.data_ptr(), FP32, 2, experts.data_ptr(), dw.data_ptr(), FP32, dx.data_ptr(), 2)
    torch.cuda.synchronize()
    d.ddp_router_destroy(h)
    assert weights.tolist() == [[0.5, 0.5], [1.0, 0.0], [0.0, 0.0]]
    assert dx.tolist() == [[0.5, -0.5], [0.0, 0.0], [0.0, 0.0]]       # w (g - mean), mean 0, 1 and nothing
