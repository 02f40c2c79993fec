"""Layer norm forward and backward through the C ABI against the 64-bit oracle.

Errors are counted, to first order, in u = 2^-24.  A sum over a row is n terms one after the other in a thread (at most 16, or a
256th of the row) and at most 12 levels of joins: |error| <= K u (sum of the terms' magnitudes), K = 28 + width / 256.  A sum
over rows: at most rows / 16 (64 at least) in a chunk, then up to 512 chunks and joins.  Roundings to a type are half a
step of it."""
import numpy as np
import pytest

from layer_cases import BF16, FP16, FP32, GUARD, TINY, U, UNIT, Rows, close, lib, torch_type, vector
from oracle import layer as ops

pytestmark = pytest.mark.gpu

PAIRS = [(FP32, FP32), (FP32, FP16), (FP32, BF16), (FP16, FP16), (BF16, BF16)]
EPS = 1e-5


def rounded_to(x, dt):
    """Bound of one rounding of x to dt."""
    return UNIT[dt] * np.abs(x) + TINY[dt] if dt != FP32 else 0.0 * np.abs(x)


def forward_bounds(x, r, gamma, beta, eps, xt, yt):
    s = x + r
    W = s.shape[1]
    K = 28 + W / 256
    y, mean, rstd = ops.norm(s, gamma, beta, eps)
    d = np.abs(s - mean[:, None])
    e_s = U * np.abs(s) * (np.abs(r) > 0).any()
    e_mean = (K + 1) * U * np.abs(s).mean(axis=1) + e_s.mean(axis=1) if np.ndim(e_s) else (K + 1) * U * np.abs(s).mean(axis=1)
    e_d = e_s + e_mean[:, None] + U * d
    # a shift of the mean by e changes the variance by e^2 alone: 2 d e sums to zero but for what the other errors leave
    e_var = (2 * d * e_d + e_d ** 2).mean(axis=1) + (K + 2) * U * (d ** 2).mean(axis=1)
    rel = 0.5 * e_var * rstd ** 2 + 4 * U
    e_y = np.abs(gamma) * rstd[:, None] * (e_d + d * (rel[:, None] + 3 * U)) + 2 * U * (np.abs(y) + np.abs(beta))
    return (s, e_s + rounded_to(s, xt)), (y, e_y + rounded_to(y, yt)), (mean, e_mean), (rstd, rel * rstd)


def check_forward(rows, width, xt, yt, pt=FP32, residual=False, gaps=(0, 0, 0, 0), shifts=(0, 0, 0, 0), params=True, stats=True, seed=0,
                  mean_of=0.3, eps=EPS):
    torch, d = lib()
    rng = np.random.default_rng(seed + width)
    x = Rows(rng.standard_normal((rows, width)) * 1.5 + mean_of, xt, gaps[0], shifts[0])
    r = Rows(rng.standard_normal((rows, width)), xt, gaps[1], shifts[1]) if residual else None
    total = Rows(np.full((rows, width), GUARD), xt, gaps[2], shifts[2]) if residual else None
    y = Rows(np.full((rows, width), GUARD), yt, gaps[3], shifts[3])
    g, gamma = vector(1 + 0.1 * rng.standard_normal(width), pt)
    b, beta = vector(0.1 * rng.standard_normal(width), pt)
    if not params:
        gamma, beta = np.ones(width), np.zeros(width)
    mean, rstd = (torch.full((rows + 2,), GUARD, device="cuda") for _ in range(2))
    h = d.ddp_layernorm_create(0, 0, width)
    torch.cuda.synchronize()
    d.ddp_layernorm_forward(h, rows, x.ptr, xt, x.stride, r.ptr if r else 0, r.stride if r else 0, g.data_ptr() if params else 0,
                            b.data_ptr() if params else None, pt, eps, total.ptr if r else 0, total.stride if r else 0, y.ptr, yt, y.stride,
                            mean[1:].data_ptr() if stats else 0, rstd[1:].data_ptr() if stats else 0)
    torch.cuda.synchronize()
    want = forward_bounds(x.held, r.held if r else np.zeros((rows, width)), gamma, beta, eps, xt, yt)
    if r:
        close(total.get(), *want[0], "sum")
        total.check_guards()
    close(y.get(), *want[1], "y")
    y.check_guards()
    x.check_guards()
    if stats:
        close(mean[1:-1].double().cpu().numpy(), *want[2], "mean")
        close(rstd[1:-1].double().cpu().numpy(), *want[3], "rstd")
        assert mean[0] == GUARD and mean[-1] == GUARD and rstd[0] == GUARD and rstd[-1] == GUARD
    d.ddp_layernorm_destroy(h)


@pytest.mark.parametrize("xt,yt", PAIRS)
@pytest.mark.parametrize("rows,width", [(1, 1), (5, 7), (3, 64), (33, 130), (9, 771), (1, 1024), (17, 1024), (6, 2050), (4, 8192), (3, 9001)])
def test_forward(xt, yt, rows, width):
    check_forward(rows, width, xt, yt)


@pytest.mark.parametrize("xt,yt", PAIRS)
@pytest.mark.parametrize("rows,width", [(1, 8), (40, 257), (70, 1024), (2, 4099), (2, 20000)])
def test_forward_with_a_residual(xt, yt, rows, width):
    check_forward(rows, width, xt, yt, residual=True)


@pytest.mark.parametrize("pt", [FP32, FP16, BF16])
@pytest.mark.parametrize("xt,yt", [(FP32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("width", [12, 515, 1024, 3000, 10000])
def test_forward_parameter_types(pt, xt, yt, width):
    check_forward(11, width, xt, yt, pt=pt)


@pytest.mark.parametrize("gaps,shifts", [((3, 0, 5, 1), (0, 1, 0, 3)), ((0, 7, 1, 0), (1, 0, 1, 1)), ((8, 8, 8, 8), (8, 8, 8, 8))])
@pytest.mark.parametrize("xt,yt", PAIRS)
@pytest.mark.parametrize("width", [5, 129, 1000])
def test_forward_strides_and_alignments(gaps, shifts, xt, yt, width):
    check_forward(21, width, xt, yt, residual=True, gaps=gaps, shifts=shifts)


@pytest.mark.parametrize("width", [24, 1024, 8500])
def test_forward_without_parameters_or_statistics(width):
    check_forward(10, width, BF16, BF16, params=False, stats=False)


@pytest.mark.parametrize("width", [16, 128, 1024, 8192, 12000])
def test_forward_far_from_zero(width):
    """Rows whose mean is 10^4 deviations: the variance comes from the differences, not from squares."""
    check_forward(4, width, FP32, FP32, mean_of=1.5e4)


def test_forward_of_equal_elements():
    torch, d = lib()
    for width in (3, 64, 1024, 8192, 9000):
        x = torch.full((5, width), 0.75, device="cuda")
        y, rstd = torch.full((5, width), GUARD, device="cuda"), torch.zeros(5, device="cuda")
        h = d.ddp_layernorm_create(0, 0, width)
        torch.cuda.synchronize()
        d.ddp_layernorm_forward(h, 5, x.data_ptr(), FP32, width, 0, 0, 0, 0, FP32, 0.25, 0, 0, y.data_ptr(), FP32, width, 0, rstd.data_ptr())
        torch.cuda.synchronize()
        assert (y == 0.0).all() and (rstd == 2.0).all()
        d.ddp_layernorm_destroy(h)


@pytest.mark.parametrize("width", [40, 1024, 8192, 9000])
def test_forward_keeps_nan_and_infinity_in_their_rows(width):
    torch, d = lib()
    x = torch.randn((8, width), device="cuda")
    clean, y = torch.zeros_like(x), torch.zeros_like(x)
    h = d.ddp_layernorm_create(0, 0, width)
    torch.cuda.synchronize()

    def forward(out):
        d.ddp_layernorm_forward(h, 8, x.data_ptr(), FP32, width, 0, 0, 0, 0, FP32, EPS, 0, 0, out.data_ptr(), FP32, width)
    forward(clean)
    torch.cuda.synchronize()
    x[2, width - 1], x[5, 0] = float("nan"), float("inf")
    forward(y)
    torch.cuda.synchronize()
    for r in range(8):
        assert torch.isnan(y[r]).all() if r in (2, 5) else torch.equal(y[r], clean[r])
    d.ddp_layernorm_destroy(h)


def backward_bounds(dy, x, mean, rstd, gamma, dsum, xt, gt, old):
    rows, W = x.shape
    K = 28 + W / 256
    dx, dgamma, dbeta = ops.norm_grad(dy, x, mean, rstd, gamma)
    xh = np.abs((x - mean[:, None]) * rstd[:, None])
    g = np.abs(dy * gamma)
    c1, c2 = g.mean(axis=1, keepdims=True), (g * xh).mean(axis=1, keepdims=True)
    e_dx = rstd[:, None] * (U * g + (K + 2) * U * c1 + (K + 8) * U * xh * c2 + 4 * U * (g + c1 + xh * c2)) + U * np.abs(dx)
    dx = dx + dsum
    e_dx = e_dx + U * np.abs(dx) + rounded_to(dx, xt)
    R = max(64, rows / 16) + 512 + 16
    out = [(dx, e_dx)]
    for value, size, before in ((dgamma, (np.abs(dy) * xh).sum(axis=0), old[0]), (dbeta, np.abs(dy).sum(axis=0), old[1])):
        value = value + before
        out.append((value, (min(R, rows + 32) + 4) * U * (size + np.abs(before)) + rounded_to(value, gt)))
    return out


def check_backward(rows, width, xt, yt, pt=FP32, gt=FP32, dsum=False, add=False, gaps=(0, 0, 0, 0), shifts=(0, 0, 0, 0), wanted="xgb", params=True,
                   seed=0, handle=None):
    torch, d = lib()
    rng = np.random.default_rng(seed + width * 3 + rows)
    x = Rows(rng.standard_normal((rows, width)) * 1.5 + 0.3, xt, gaps[0], shifts[0])
    dy = Rows(rng.standard_normal((rows, width)), yt, gaps[1], shifts[1])
    more = Rows(rng.standard_normal((rows, width)), xt, gaps[2], shifts[2]) if dsum else None
    dx = Rows(np.full((rows, width), GUARD), xt, gaps[3], shifts[3])
    g, gamma = vector(1 + 0.1 * rng.standard_normal(width), pt)
    if not params:
        gamma = np.ones(width)
    _, mean, rstd = ops.norm(x.held, 1.0, 0.0, EPS)
    mean_on, mean = vector(mean, FP32)
    rstd_on, rstd = vector(rstd, FP32)
    dgamma, old_gamma = vector(rng.standard_normal(width), gt)
    dbeta, old_beta = vector(rng.standard_normal(width), gt)
    h = handle or d.ddp_layernorm_create(0, 0, width)
    torch.cuda.synchronize()
    d.ddp_layernorm_backward(h, rows, dy.ptr, yt, dy.stride, x.ptr, xt, x.stride, mean_on.data_ptr(), rstd_on.data_ptr(),
                             g.data_ptr() if params else 0, pt, more.ptr if dsum else 0, more.stride if dsum else 0,
                             dx.ptr if "x" in wanted else 0, dx.stride, add, dgamma.data_ptr() if "g" in wanted else 0,
                             dbeta.data_ptr() if "b" in wanted else 0, gt)
    torch.cuda.synchronize()
    old = (old_gamma, old_beta) if add else (np.zeros(width), np.zeros(width))
    want = backward_bounds(dy.held, x.held, mean, rstd, gamma, more.held if dsum else 0.0 * x.held, xt, gt, old)
    if "x" in wanted:
        close(dx.get(), *want[0], "dx")
    dx.check_guards()
    for flag, got, before, w in (("g", dgamma, old_gamma, want[1]), ("b", dbeta, old_beta, want[2])):
        got = got.double().cpu().numpy()
        if flag in wanted:
            close(got, *w, flag)
        else:
            assert (got == before).all()
    if handle is None:
        d.ddp_layernorm_destroy(h)
    return dx.buf.clone(), dgamma.clone(), dbeta.clone()


@pytest.mark.parametrize("xt,yt", PAIRS)
@pytest.mark.parametrize("rows,width", [(1, 1), (5, 7), (3, 64), (700, 130), (9, 771), (1, 1024), (2100, 1024), (6, 2050), (4, 8192), (3, 9001)])
def test_backward(xt, yt, rows, width):
    check_backward(rows, width, xt, yt)


@pytest.mark.parametrize("xt,yt", PAIRS)
@pytest.mark.parametrize("rows,width", [(1, 8), (400, 257), (70, 1024), (200, 4099), (66, 20000)])
def test_backward_added_with_what_flows_along_the_sum(xt, yt, rows, width):
    check_backward(rows, width, xt, yt, dsum=True, add=True)


@pytest.mark.parametrize("pt", [FP32, FP16, BF16])
@pytest.mark.parametrize("gt", [FP32, FP16, BF16])
@pytest.mark.parametrize("width", [12, 515, 1024, 10000])
def test_backward_parameter_types(pt, gt, width):
    check_backward(45, width, BF16, BF16, pt=pt, gt=gt, add=gt == FP16)


@pytest.mark.parametrize("gaps,shifts", [((3, 0, 5, 1), (0, 1, 0, 3)), ((0, 7, 1, 0), (1, 0, 1, 1)), ((8, 8, 8, 8), (8, 8, 8, 8))])
@pytest.mark.parametrize("xt,yt", PAIRS)
@pytest.mark.parametrize("width", [5, 129, 1000])
def test_backward_strides_and_alignments(gaps, shifts, xt, yt, width):
    check_backward(130, width, xt, yt, dsum=True, gaps=gaps, shifts=shifts)


@pytest.mark.parametrize("wanted", ["", "x", "g", "b", "gb", "xg", "xb"])
@pytest.mark.parametrize("width", [72, 1024, 9000])
def test_backward_of_some_alone(wanted, width):
    check_backward(77, width, BF16, BF16, wanted=wanted, params=False)


@pytest.mark.parametrize("rows,width", [(70001, 16), (40003, 64), (9001, 520), (3000, 5000)])
def test_backward_of_many_rows(rows, width):
    check_backward(rows, width, FP32, FP32)


def test_backward_of_no_rows():
    torch, d = lib()
    for width in (5, 1024, 9000):
        h = d.ddp_layernorm_create(0, 0, width)
        dgamma, dbeta = torch.full((width,), GUARD, device="cuda"), torch.full((width,), GUARD, device="cuda")
        torch.cuda.synchronize()
        for add, left in ((True, GUARD), (False, 0.0)):
            d.ddp_layernorm_backward(h, 0, 0, FP32, width, 0, FP32, width, 0, 0, 0, FP32, 0, 0, 0, width, add, dgamma.data_ptr(),
                                     dbeta.data_ptr(), FP32)
            torch.cuda.synchronize()
            assert (dgamma == left).all() and (dbeta == left).all()
        d.ddp_layernorm_forward(h, 0, 0, FP32, width, 0, 0, 0, 0, FP32, EPS, 0, 0, 0, FP32, width)
        d.ddp_layernorm_destroy(h)


@pytest.mark.parametrize("rows,width", [(5000, 64), (3000, 1024), (500, 9000)])
def test_same_bits_again(rows, width):
    torch, d = lib()
    h = d.ddp_layernorm_create(0, 0, width)
    first = check_backward(rows, width, BF16, BF16, handle=h)
    check_backward(rows // 3, width, BF16, BF16, handle=h, seed=9)      # another call between leaves nothing behind
    for a, b in zip(first, check_backward(rows, width, BF16, BF16, handle=h)):
        assert torch.equal(a, b)
    d.ddp_layernorm_destroy(h)


def test_rows_past_32_bits():
    """4.3 GB of x, y and dx: the offsets of the last rows need more than 32 bits."""
    torch, d = lib()
    rows, width = 2_100_000, 1024
    x = torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda")
    x[:, ::2] = 1.0
    y = torch.zeros_like(x)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    dgamma, dbeta = torch.zeros(width, device="cuda"), torch.zeros(width, device="cuda")
    h = d.ddp_layernorm_create(0, 0, width)
    torch.cuda.synchronize()
    d.ddp_layernorm_forward(h, rows, x.data_ptr(), BF16, width, 0, 0, 0, 0, FP32, 0.0, 0, 0, y.data_ptr(), BF16, width, mean.data_ptr(),
                            rstd.data_ptr())
    torch.cuda.synchronize()
    assert (mean == 0.5).all() and (rstd == 2.0).all() and (y[-1, ::2] == 1.0).all() and (y[-1, 1::2] == -1.0).all()
    assert (y[:, 0] == 1.0).all() and (y[:, -1] == -1.0).all()
    dx = torch.full_like(x, GUARD)
    # dy = y: all of it is along what the norm takes out, dgamma = rows, dbeta = +-rows
    d.ddp_layernorm_backward(h, rows, y.data_ptr(), BF16, width, x.data_ptr(), BF16, width, mean.data_ptr(), rstd.data_ptr(), 0, FP32, 0, 0,
                             dx.data_ptr(), width, False, dgamma.data_ptr(), dbeta.data_ptr(), FP32)
    torch.cuda.synchronize()
    assert (dx == 0.0).all()
    assert (dgamma == rows).all() and (dbeta[::2] == rows).all() and (dbeta[1::2] == -rows).all()
    d.ddp_layernorm_destroy(h)


def test_on_another_stream_and_replayed():
    """Forward and backward captured into a graph on a stream of their own, replayed between eager work."""
    torch, d = lib()
    rows, width = 3000, 1024
    stream = torch.cuda.Stream()
    h = d.ddp_layernorm_create(0, stream.cuda_stream, width)
    x = torch.randn((rows, width), device="cuda").bfloat16()
    gamma, beta = torch.rand(width, device="cuda"), torch.rand(width, device="cuda")
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    mean, rstd, dgamma, dbeta = (torch.zeros(n, device="cuda") for n in (rows, rows, width, width))
    torch.cuda.synchronize()

    def both():
        d.ddp_layernorm_forward(h, rows, x.data_ptr(), BF16, width, 0, 0, gamma.data_ptr(), beta.data_ptr(), FP32, EPS, 0, 0, y.data_ptr(), BF16,
                                width, mean.data_ptr(), rstd.data_ptr())
        d.ddp_layernorm_backward(h, rows, y.data_ptr(), BF16, width, x.data_ptr(), BF16, width, mean.data_ptr(), rstd.data_ptr(),
                                 gamma.data_ptr(), FP32, 0, 0, dx.data_ptr(), width, False, dgamma.data_ptr(), dbeta.data_ptr(), FP32)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        both()
        stream.synchronize()
        graph.capture_begin()
        both()
        graph.capture_end()
    for seed in range(4):
        with torch.cuda.stream(stream):
            x.copy_(torch.randn((rows, width), generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
            both()
            stream.synchronize()
            want = [t.clone() for t in (y, dx, mean, rstd, dgamma, dbeta)]
            for t in (y, dx, mean, rstd, dgamma, dbeta):
                t.fill_(GUARD)
            graph.replay()
            stream.synchronize()
            for t, w in zip((y, dx, mean, rstd, dgamma, dbeta), want):
                assert torch.equal(t, w)
    torch.cuda.synchronize()
    d.ddp_layernorm_destroy(h)


@pytest.mark.parametrize("xt,yt", [(FP32, FP32), (FP32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("rows,width", [(9000, 1024), (9001, 515), (40001, 64), (150001, 16), (2500, 2100), (3001, 4000), (600, 8100)])
def test_forward_of_many_rows(xt, yt, rows, width):
    """More rows than the launch has teams, results that go past the caches."""
    check_forward(rows, width, xt, yt, residual=True)


@pytest.mark.parametrize("xt,yt", [(FP32, FP32), (FP32, FP16), (BF16, BF16)])
@pytest.mark.parametrize("rows,width", [(300, 16), (301, 24), (99, 32), (50, 48), (70, 300), (70, 512), (41, 1500), (41, 2048), (9, 4096), (5, 6000), (5, 16384),
                                        (3, 16385)])
def test_both_ways_of_every_team(xt, yt, rows, width):
    check_forward(rows, width, xt, yt, residual=True, gaps=(1, 0, 3, 2))
    check_backward(rows, width, xt, yt, dsum=True, gaps=(0, 3, 1, 2))


@pytest.mark.parametrize("rows,width", [(5000, 1500), (70000, 24), (900, 10048)])
def test_backward_of_more_rows_than_teams(rows, width):
    check_backward(rows, width, BF16, BF16, dsum=True, add=True)
    check_backward(rows, width, FP32, BF16, wanted="gb")


def test_two_handles_at_once():
    """Handles on two streams, their calls in turn: workspaces of their own."""
    torch, d = lib()
    rows, width = 4000, 1024
    streams = [torch.cuda.Stream() for _ in range(2)]
    handles = [d.ddp_layernorm_create(0, s.cuda_stream, width) for s in streams]
    gen = torch.Generator("cuda").manual_seed(3)
    x, dy = (torch.randn((2, rows, width), generator=gen, device="cuda") for _ in range(2))
    mean, rstd = x.mean(2), x.var(2, unbiased=False).rsqrt()
    out = torch.zeros((8, 2, 2, width), device="cuda")
    torch.cuda.synchronize()
    for turn in range(8):
        for k in range(2):
            d.ddp_layernorm_backward(handles[k], rows, dy[k].data_ptr(), FP32, width, x[k].data_ptr(), FP32, width, mean[k].data_ptr(), rstd[k].data_ptr(), 0,
                                     FP32, 0, 0, 0, 0, False, out[turn, k, 0].data_ptr(), out[turn, k, 1].data_ptr(), FP32)
    torch.cuda.synchronize()
    assert (out == out[0]).all()
    for k in range(2):
        want = (dy[k].double() * ((x[k].double() - mean[k].double()[:, None]) * rstd[k].double()[:, None])).sum(0)
        assert (out[0, k, 0].double() - want).abs().max() < 1e-3
    for h in handles:
        d.ddp_layernorm_destroy(h)


@pytest.mark.parametrize("width", [5, 24, 70, 515, 1024, 1500, 3001, 6000, 10001, 17000])
@pytest.mark.parametrize("dt", [FP32, BF16])
def test_in_place(width, dt):
    """The sum over x or over the residual, dx over what flows along the sum: the same bits as apart."""
    torch, d = lib()
    rows = 50
    gen = torch.Generator("cuda").manual_seed(width)
    x, r, dy = (torch.randn((rows, width), generator=gen, device="cuda").to(torch_type(dt)) for _ in range(3))
    gamma, beta = (torch.randn(width, generator=gen, device="cuda") for _ in range(2))
    h = d.ddp_layernorm_create(0, 0, width)

    def forward(x, r, total):
        y, mean, rstd = torch.zeros_like(x), torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        d.ddp_layernorm_forward(h, rows, x.data_ptr(), dt, width, r.data_ptr(), width, gamma.data_ptr(), beta.data_ptr(), FP32, EPS, total.data_ptr(), width,
                                y.data_ptr(), dt, width, mean.data_ptr(), rstd.data_ptr())
        return y, mean, rstd, total

    def backward(along, dx):
        dgamma, dbeta = torch.zeros(width, device="cuda"), torch.zeros(width, device="cuda")
        d.ddp_layernorm_backward(h, rows, dy.data_ptr(), dt, width, x.data_ptr(), dt, width, mean.data_ptr(), rstd.data_ptr(), gamma.data_ptr(), FP32,
                                 along.data_ptr(), width, dx.data_ptr(), width, False, dgamma.data_ptr(), dbeta.data_ptr(), FP32)
        return dx, dgamma, dbeta
    torch.cuda.synchronize()
    apart = forward(x, r, torch.zeros_like(x))
    _, mean, rstd, _ = apart
    for which in (0, 1):
        ins = [x.clone(), r.clone()]
        for a, b in zip(forward(*ins, ins[which]), apart):
            assert torch.equal(a, b)
    want = backward(r, torch.zeros_like(x))
    along = r.clone()
    for a, b in zip(backward(along, along), want):
        assert torch.equal(a, b)
    d.ddp_layernorm_destroy(h)


@pytest.mark.parametrize("rows,width", [(1, 64), (8, 256), (30, 500), (33, 512), (33, 513), (200, 128), (2000, 24), (129, 17)])
def test_backward_of_few_rows_again_and_again(rows, width):
    """Where the last block joins the sums: whole numbers, so that every order of them has the same sum; other sizes on the same handle and replays of
    a graph in between, and what is added to."""
    torch, d = lib()
    gen = torch.Generator("cuda").manual_seed(width)
    stream = torch.cuda.Stream()
    h = d.ddp_layernorm_create(0, stream.cuda_stream, width)
    many = 40000
    dy = torch.randint(-2, 3, (many, width), generator=gen, device="cuda").float()
    x = torch.randint(-2, 3, (many, width), generator=gen, device="cuda").float()
    mean, rstd, dx = torch.zeros(many, device="cuda"), torch.ones(many, device="cuda"), torch.empty_like(x)
    dgamma, dbeta = torch.zeros(width, device="cuda"), torch.zeros(width, device="cuda")
    torch.cuda.synchronize()

    def call(n, add):
        d.ddp_layernorm_backward(h, n, dy.data_ptr(), FP32, width, x.data_ptr(), FP32, width, mean.data_ptr(), rstd.data_ptr(), 0, FP32, 0, 0, dx.data_ptr(),
                                 width, add, dgamma.data_ptr(), dbeta.data_ptr(), FP32)

    def want(n):
        return (dy[:n].double() * x[:n].double()).sum(0).float(), dy[:n].double().sum(0).float()

    few, one, all_of_them = want(rows), want(1), want(many)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        call(rows, False)
        stream.synchronize()
        graph.capture_begin()
        call(rows, True)
        graph.capture_end()
        for turn in range(50):
            call(rows, False)
            assert torch.equal(dgamma, few[0]) and torch.equal(dbeta, few[1]), turn
            call(1, True)
            assert torch.equal(dgamma, few[0] + one[0]) and torch.equal(dbeta, few[1] + one[1]), turn
            graph.replay()
            assert torch.equal(dgamma, 2 * few[0] + one[0]) and torch.equal(dbeta, 2 * few[1] + one[1]), turn
            if turn % 10 == 0:
                call(many, False)
                assert torch.equal(dgamma, all_of_them[0]) and torch.equal(dbeta, all_of_them[1]), turn
        stream.synchronize()
    torch.cuda.synchronize()
    d.ddp_layernorm_destroy(h)
