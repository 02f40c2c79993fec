"""Routing to experts, its gradient and the balance bias through the C ABI against the 64-bit oracle.

Choices are compared for equality: they are made as binary64 has the keys, and equal keys (equal logits, equal biases) go to the lower index.
Weights in binary32: exp(x) of a rounded x is off by |x| u and 2 u of its own, a sum of n terms by (n / 16 + 12) u, so that
a weight is off by R u of itself, R = 2 (largest difference of logits) + experts / 16 + 40.  The gradient's terms are products of such
weights: twice R u of the terms' magnitudes."""
import numpy as np
import pytest

from layer_cases import BF16, FP16, FP32, GUARD, TINY, U, UNIT, Rows, close, lib, torch_type, vector
from oracle import layer as ops

pytestmark = pytest.mark.gpu

SOFTMAX, SIGMOID = 0, 1
KINDS = [(4, 2, 1, 1, 1), (1, 1, 1, 1, 2), (64, 2, 1, 1, 1), (60, 4, 1, 1, 1), (128, 6, 4, 2, 2), (256, 8, 8, 4, 2), (255, 9, 5, 2, 1), (160, 6, 8, 3, 1),
         (1024, 64, 64, 7, 2), (7, 7, 1, 1, 1), (512, 16, 1, 1, 1), (33, 3, 11, 2, 2), (8, 3, 8, 5, 2)]


def spread(x):
    x = np.where(np.isfinite(x), x, 0.0)
    return np.maximum(x.max(axis=1) - x.min(axis=1), np.abs(x).max(axis=1))


def check_route(tokens, kind, score, renormalise, dt=FP32, wt=FP32, scale=2.5, bias=True, gap=0, shift=0, add=False, seed=0, logits=None, stats=True,
                handle=None, times=1):
    torch, d = lib()
    E, k, groups, kept, top = kind
    rng = np.random.default_rng(seed + E)
    x = Rows(np.tile(rng.standard_normal((tokens, E)) * 1.5 if logits is None else logits, (times, 1)), dt, gap, shift)
    few, tokens = tokens, tokens * times
    b = (rng.integers(-40, 41, E) * np.float32(1e-3)).astype(np.float32) if bias is True else bias
    b_on = torch.from_numpy(b).cuda() if b is not None and bias is not False else None
    experts = torch.full((tokens + 1, k), 99, dtype=torch.int32, device="cuda")
    weights = torch.full((tokens + 1, k), GUARD, dtype=torch_type(wt), device="cuda")
    counts = torch.arange(E + 1, dtype=torch.int32, device="cuda")
    h = handle or d.ddp_router_create(0, 0, E, k, groups, kept, top, score, renormalise, scale)
    torch.cuda.synchronize()
    d.ddp_router_route(h, tokens, x.ptr, dt, x.stride, b_on.data_ptr() if b_on is not None else 0, experts.data_ptr(), weights.data_ptr(), wt,
                       counts.data_ptr() if stats else 0, add)
    torch.cuda.synchronize()
    want, w = ops.route(x.held[:few], b if b_on is not None else np.zeros(E), k, groups, kept, top, score, renormalise, scale)
    want, w = np.tile(want, (times, 1)), np.tile(w, (times, 1))
    got = experts[:-1].cpu().numpy()
    assert (got == want).all(), (np.argwhere(got != want)[:3].tolist(), got[(got != want).any(1)][:2], want[(got != want).any(1)][:2])
    R = (2 * spread(x.held) + E / 16 + 40)[:, None]
    close(weights[:-1].double().cpu().numpy(), w, R * U * np.abs(w) + UNIT[wt] * np.abs(w) + max(TINY[wt], 2.0 ** -126), "weights")
    assert (experts[-1] == 99).all() and (weights[-1] == GUARD).all()
    load = np.bincount(want[want >= 0], minlength=E) if stats else np.arange(E)
    if add and stats:
        load = load + np.arange(E)
    assert (counts[:-1].cpu().numpy() == load).all() and counts[-1] == E
    if handle is None:
        d.ddp_router_destroy(h)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route(kind, score, renormalise):
    check_route(150, kind, score, renormalise)


@pytest.mark.parametrize("dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("wt", [FP32, FP16, BF16])
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_route_types(dt, wt, score):
    check_route(90, (64, 6, 4, 2, 2), score, True, dt, wt, gap=3, shift=1, add=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_route_equal_keys(kind, score):
    """Logits of few values: most keys are equal to others, and go to the lower index, among groups too."""
    rng = np.random.default_rng(kind[0])
    logits = rng.integers(-2, 3, (120, kind[0])) * 0.5
    logits[7] = 0.0
    check_route(120, kind, score, True, BF16, logits=logits, bias=False)
    check_route(120, kind, score, False, FP32, logits=logits, bias=(rng.integers(0, 2, kind[0]) * 0.125).astype(np.float32))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_route_nearly_equal_keys(kind, score):
    """Logits one step of binary32 apart: binary64 tells their keys apart, binary32 mostly does not."""
    rng = np.random.default_rng(kind[0] + 1)
    logits = (1.0 + rng.integers(0, 4 * kind[0], (80, kind[0])) * 2.0 ** -23).astype(np.float32).astype(np.float64)
    check_route(80, kind, score, True, logits=logits, bias=False)
    check_route(80, kind, score, True, logits=logits, bias=np.full(kind[0], 0.37, dtype=np.float32))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_route_masked_experts(kind, score):
    rng = np.random.default_rng(kind[0])
    logits = rng.standard_normal((64, kind[0]))
    logits[rng.random(logits.shape) < 0.5] = -np.inf
    logits[3] = -np.inf
    logits[5] = np.nan
    logits[9, 0] = np.nan
    logits[11, -1] = np.inf
    logits[13] = -1e30
    logits[15] = 1e30
    check_route(64, kind, score, True, logits=logits)
    check_route(64, kind, score, False, logits=logits, bias=False)
    bias = rng.standard_normal(kind[0]).astype(np.float32)
    bias[::3] = -np.inf
    bias[1::5] = np.nan
    check_route(64, kind, score, True, logits=logits, bias=bias)


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("tokens", [0, 1, 2, 3, 15, 16, 17, 4099])
def test_route_numbers_of_tokens(score, tokens):
    check_route(tokens, (64, 6, 8, 3, 2), score, True, BF16)
    check_route(tokens, (40, 2, 1, 1, 1), score, True, FP32, stats=tokens % 2 == 0)


def test_route_wide_range():
    rng = np.random.default_rng(1)
    logits = rng.standard_normal((50, 96)) * 60.0
    check_route(50, (96, 8, 1, 1, 1), SOFTMAX, True, logits=logits, bias=False)
    check_route(50, (96, 8, 1, 1, 1), SIGMOID, True, logits=logits, bias=False)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("times", [1, 1000])
def test_route_biases_at_the_end_of_binary32(kind, score, times):
    """As masks (the lowest value), and as what is chosen first."""
    E, most = kind[0], np.finfo(np.float32).max
    rng = np.random.default_rng(E)
    logits = rng.standard_normal((40, E))
    for values in ([0.0, -most], [0.0, 0.25, most, -most], [most * 0.75, -most * 0.75, -np.inf]):
        bias = rng.choice(np.array(values, dtype=np.float32), E)
        check_route(40, kind, score, True, logits=logits, bias=bias, times=times)


def far_below(rng, tokens, E):
    """Logits of which every second one is some hundred below the others, and what makes those the chosen ones."""
    logits = rng.standard_normal((tokens, E)) * 2.0
    logits[:, ::2] -= 110.0
    bias = np.zeros(E, dtype=np.float32)
    bias[::2] = 8.0 + rng.integers(0, 40, (E + 1) // 2) * 0.125
    return logits, bias


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("times", [1, 1000])
def test_route_scores_below_binary32(kind, score, times):
    """The chosen scores and their sum leave binary32, their quotients do not."""
    logits, bias = far_below(np.random.default_rng(kind[0]), 40, kind[0])
    logits[1] -= 100.0
    check_route(40, kind, score, True, logits=logits, bias=bias, times=times)
    check_route(40, kind, score, False, logits=logits, bias=bias, times=times)


def check_grad(tokens, kind, score, renormalise, dt=FP32, wt=FP32, scale=2.5, gap=0, shift=0, seed=0, experts=None, logits=None):
    torch, d = lib()
    E, k = kind[:2]
    rng = np.random.default_rng(seed + E)
    x = Rows(rng.standard_normal((tokens, E)) * 1.5 if logits is None else logits, dt, gap, shift)
    if experts is None:
        experts = np.argsort(rng.random((tokens, E)), axis=1)[:, :k]
    at = torch.from_numpy(np.ascontiguousarray(experts)).int().cuda()
    dw = Rows(rng.standard_normal((tokens, k)), wt)
    dx = Rows(np.full((tokens, E), GUARD), dt, gap + 2, shift)
    h = d.ddp_router_create(0, 0, *kind, score, renormalise, scale)
    torch.cuda.synchronize()
    d.ddp_router_grad(h, tokens, x.ptr, dt, x.stride, at.data_ptr(), dw.ptr, wt, dx.ptr, dx.stride)
    torch.cuda.synchronize()
    want, magnitude = ops.route_grad(x.held, experts, dw.held, score, renormalise, scale)
    R = (2 * spread(x.held) + E / 16 + 40)[:, None]
    close(dx.get(), want, 4 * R * U * magnitude + UNIT[dt] * np.abs(want) + max(TINY[dt], 2.0 ** -126), "dlogits")
    dx.check_guards()
    d.ddp_router_destroy(h)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("renormalise", [False, True])
def test_grad(kind, score, renormalise):
    check_grad(150, kind, score, renormalise)


@pytest.mark.parametrize("dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("wt", [FP32, FP16, BF16])
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_grad_types(dt, wt, score):
    check_grad(90, (60, 6, 4, 2, 2), score, True, dt, wt, gap=3, shift=1)


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("tokens", [0, 1, 2, 3, 15, 16, 17, 4099])
def test_grad_numbers_of_tokens(score, tokens):
    check_grad(tokens, (64, 6, 8, 3, 2), score, True, BF16)


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("renormalise", [False, True])
def test_grad_of_places_left_over(score, renormalise):
    """Indices of no expert take no part, a token without any gets zeros, one that is named twice counts twice; masked logits get zeros."""
    rng = np.random.default_rng(4)
    experts = np.argsort(rng.random((40, 70)), axis=1)[:, :5]
    experts[::3, 3:] = -1
    experts[4] = -1
    experts[7] = [3, 70, 3, -5, 2 ** 31 - 1]
    experts[8] = [69, 69, 69, 69, 69]
    logits = rng.standard_normal((40, 70))
    logits[::3, 1::2] = -np.inf
    experts[::3, :3] = [0, 2, 4]
    check_grad(40, (70, 5, 1, 1, 1), score, renormalise, experts=experts, logits=logits)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("renormalise", [False, True])
def test_grad_of_scores_below_binary32(kind, score, renormalise):
    E, k = kind[:2]
    rng = np.random.default_rng(E)
    logits = far_below(rng, 40, E)[0]
    experts = np.stack([rng.permutation(np.arange(0, E, 2))[:k] for _ in range(40)])
    experts = np.pad(experts, ((0, 0), (0, k - experts.shape[1])), constant_values=-1)
    experts[::7, 0] = E - 1 - (E - 1) % 2
    check_grad(40, kind, score, renormalise, logits=logits, experts=experts)


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_grad_of_large_logits(score):
    rng = np.random.default_rng(5)
    check_grad(30, (50, 4, 1, 1, 1), score, True, logits=rng.standard_normal((30, 50)) * 20.0)


@pytest.mark.parametrize("replicas,experts", [(1, 1), (1, 8), (3, 60), (8, 256), (64, 1024)])
def test_balance(replicas, experts):
    torch, d = lib()
    rng = np.random.default_rng(experts)
    counts = rng.integers(0, 5, (replicas, experts))
    counts[:, experts // 2] = 2 ** 31 - 1 if experts > 8 else 2
    bias = rng.standard_normal(experts).astype(np.float32)
    on, b = torch.from_numpy(counts).int().cuda(), torch.from_numpy(bias).cuda()
    out = torch.full((experts + 1,), GUARD, device="cuda")
    h = d.ddp_router_create(0, 0, experts, 1)
    torch.cuda.synchronize()
    d.ddp_router_balance(h, replicas, on.data_ptr(), 1e-3, b.data_ptr(), out.data_ptr())
    torch.cuda.synchronize()
    want = torch.from_numpy(ops.balance(counts, bias, 1e-3))
    assert torch.equal(out[:-1].cpu(), want) and out[-1] == GUARD
    d.ddp_router_balance(h, replicas, on.data_ptr(), 1e-3, b.data_ptr(), b.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(b.cpu(), want)
    d.ddp_router_destroy(h)


def test_tokens_past_32_bits():
    """Logits of 4.4 GB: the offsets of the last tokens need more than 32 bits."""
    torch, d = lib()
    T, E, k = 17_000_000, 130, 1
    x = torch.zeros((T, E), dtype=torch.bfloat16, device="cuda")
    x[:, 5] = 1.0
    x[-1, 5], x[-1, 129] = 0.0, 1.0
    experts = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    weights, counts = torch.zeros((T, k), device="cuda"), torch.zeros(E, dtype=torch.int32, device="cuda")
    h = d.ddp_router_create(0, 0, E, k, score=SIGMOID)
    torch.cuda.synchronize()
    d.ddp_router_route(h, T, x.data_ptr(), BF16, E, 0, experts.data_ptr(), weights.data_ptr(), FP32, counts.data_ptr())
    torch.cuda.synchronize()
    assert counts[5] == T - 1 and counts[129] == 1 and counts.sum() == T and experts[-1, 0] == 129 and (weights == 1.0).all()
    d.ddp_router_destroy(h)
    h = d.ddp_router_create(0, 0, E, k, score=SIGMOID, renormalise=False)
    weights.fill_(1.0)
    torch.cuda.synchronize()
    d.ddp_router_grad(h, T, x.data_ptr(), BF16, E, experts.data_ptr(), weights.data_ptr(), FP32, x.data_ptr(), E)
    torch.cuda.synchronize()
    s = 1 / (1 + np.exp(-1.0))
    assert abs(x[-1, 129].item() - s * (1 - s)) < 2 ** -8 and (x[:-1, 5] == x[-1, 129]).all() and (x[-1, :129] == 0).all()
    assert x.count_nonzero() == T
    d.ddp_router_destroy(h)


def test_on_another_stream_and_replayed():
    torch, d = lib()
    T, E, k = 3000, 64, 4
    stream = torch.cuda.Stream()
    h = d.ddp_router_create(0, stream.cuda_stream, E, k, 8, 4, 2, SIGMOID, True, 2.5)
    x, dx = torch.zeros((T, E), device="cuda"), torch.zeros((T, E), device="cuda")
    bias, moved = torch.zeros(E, device="cuda"), torch.zeros(E, device="cuda")
    experts, counts = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros(E, dtype=torch.int32, device="cuda")
    weights = torch.zeros((T, k), device="cuda")
    torch.cuda.synchronize()

    def all_of_it():
        d.ddp_router_route(h, T, x.data_ptr(), FP32, E, bias.data_ptr(), experts.data_ptr(), weights.data_ptr(), FP32, counts.data_ptr())
        d.ddp_router_grad(h, T, x.data_ptr(), FP32, E, experts.data_ptr(), weights.data_ptr(), FP32, dx.data_ptr(), E)
        d.ddp_router_balance(h, 1, counts.data_ptr(), 0.01, bias.data_ptr(), moved.data_ptr())

    results = experts, weights, counts, dx, moved
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        all_of_it()
        stream.synchronize()
        graph.capture_begin()
        all_of_it()
        graph.capture_end()
        for seed in range(4):
            x.copy_(torch.randn((T, E), generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
            all_of_it()
            stream.synchronize()
            want = [t.clone() for t in results]
            for t in results:
                t.fill_(99)
            graph.replay()
            stream.synchronize()
            for t, w in zip(results, want):
                assert torch.equal(t, w)
    torch.cuda.synchronize()
    d.ddp_router_destroy(h)


BIG = [(256, 8, 8, 4, 2, SIGMOID, FP32, True), (256, 8, 1, 1, 1, SOFTMAX, BF16, False), (64, 2, 1, 1, 1, SOFTMAX, BF16, True), (60, 4, 1, 1, 1, SIGMOID, FP16, True),
       (1000, 16, 1, 1, 1, SOFTMAX, FP32, True), (8, 3, 2, 1, 2, SIGMOID, BF16, False), (160, 6, 8, 3, 1, SOFTMAX, FP32, True), (130, 40, 1, 1, 1, SIGMOID, BF16, True),
       (24, 2, 12, 6, 2, SIGMOID, FP32, True), (512, 4, 64, 8, 2, SOFTMAX, BF16, False)]


@pytest.mark.parametrize("E,k,groups,kept,top,score,dt,biased", BIG)
def test_many_tokens_as_few(E, k, groups, kept, top, score, dt, biased):
    """Long calls leave the tokens whose keys come near each other to a second kernel: they choose what short calls do (which are
    compared with the oracle above), and count the same, at every call."""
    torch, d = lib()
    T, some = 70000, 700
    gen = torch.Generator("cuda").manual_seed(E)
    x = (torch.randn((T, E), generator=gen, device="cuda") * 1.5).to(torch_type(dt))
    x[::97, ::2] = x[::97, 1::2]                          # pairs of equal logits
    x[5::101] = (x[5::101].float() * 1e-3).to(x.dtype)    # many that are nearly equal
    x[7::103, : E // 2] = -float("inf")
    bias = (torch.randint(-40, 41, (E,), generator=gen, device="cuda") * 1e-3) if biased else None
    h = d.ddp_router_create(0, 0, E, k, groups, kept, top, score, True, 2.5)
    big, small = ((torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda"),
                   torch.full((E,), 5, dtype=torch.int32, device="cuda")) for _ in range(2))
    torch.cuda.synchronize()

    def route(out, a, n, add):
        d.ddp_router_route(h, n, x[a:a + n].data_ptr(), dt, E, bias.data_ptr() if biased else 0, out[0][a:].data_ptr(), out[1][a:].data_ptr(), FP32,
                           out[2].data_ptr(), add)
    for a in range(0, T, some):
        route(small, a, some, a > 0)
    for add in (False, False, True):
        big[0].fill_(-2)
        route(big, 0, T, add)
    torch.cuda.synchronize()
    assert torch.equal(big[0], small[0])
    assert ((big[1] - small[1]).abs() <= 2 * (2 * 20 + E / 16 + 40) * U * small[1]).all()
    load = torch.bincount(small[0][small[0] >= 0], minlength=E)
    assert torch.equal(small[2].long(), load) and torch.equal(big[2].long(), 2 * load)
    d.ddp_router_destroy(h)


@pytest.mark.parametrize("experts,chosen", [(143, 14), (64, 2), (1024, 8), (20, 20), (6, 1)])
@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
def test_grad_of_many_tokens_as_few(experts, chosen, score):
    torch, d = lib()
    T, some = 60000, 1500
    gen = torch.Generator("cuda").manual_seed(experts)
    x = torch.randn((T, experts), generator=gen, device="cuda").bfloat16()
    at = torch.rand((T, experts), generator=gen, device="cuda").topk(chosen, dim=1).indices.int()
    at[::7, -1] = -1
    dw = torch.randn((T, chosen), generator=gen, device="cuda")
    h = d.ddp_router_create(0, 0, experts, chosen, score=score)
    big, small = (torch.full((T, experts), GUARD, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    torch.cuda.synchronize()

    def grad(out, a, n):
        d.ddp_router_grad(h, n, x[a:].data_ptr(), BF16, experts, at[a:].data_ptr(), dw[a:].data_ptr(), FP32, out[a:].data_ptr(), experts)
    grad(big, 0, T)
    for a in range(0, T, some):
        grad(small, a, some)
    torch.cuda.synchronize()
    assert torch.equal(big, small)
    grad(x, 0, T)                                         # over the logits
    torch.cuda.synchronize()
    assert torch.equal(big, x)
    d.ddp_router_destroy(h)
