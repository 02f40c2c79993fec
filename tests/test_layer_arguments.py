"""What the calls inside a layer refuse, on handles without a device, and the binding's own checks."""
import pytest

FP32, FP16, BF16 = 0, 1, 2
BIG = 1 << 24


@pytest.fixture(scope="module")
def d():
    import paper_2006_15704_amd as lib
    return lib


def refused(d, code, call, *args):
    with pytest.raises(d.DdpError) as e:
        call(*args)
    assert e.value.code == code, e.value
    assert len(str(e.value)) > len(f"ddp error {code}: "), "no text"


def changed(args, **at):
    """args (a dict in the order of the call) with some of them replaced."""
    assert set(at) <= set(args)
    return list({**args, **at}.values())


def test_handles(d):
    for make in (lambda dev: d.ddp_layernorm_create(dev, 0, 8), lambda dev: d.ddp_position_bias_create(dev, 0, 2, 32, 16, 128, False),
                 lambda dev: d.ddp_router_create(dev, 0, 8, 2)):
        refused(d, d.DDP_ERR_ARG, make, -2)
        refused(d, d.DDP_ERR_HIP, make, 4096)
    for width, code in ((0, d.DDP_ERR_ARG), (-1, d.DDP_ERR_ARG), ((1 << 20) + 1, d.DDP_ERR_UNSUPPORTED)):
        refused(d, code, d.ddp_layernorm_create, d.DDP_DEVICE_NONE, 0, width)
    for args, code in (((0, 32, 16, 128, False), d.DDP_ERR_ARG), ((2, 0, 1, 128, False), d.DDP_ERR_ARG), ((2, 32, 0, 128, False), d.DDP_ERR_ARG),
                       ((2, 32, 33, 128, False), d.DDP_ERR_ARG), ((2, 32, 17, 128, True), d.DDP_ERR_ARG), ((2, 31, 4, 128, True), d.DDP_ERR_ARG),
                       ((2, 32, 16, 16, False), d.DDP_ERR_ARG), ((2, 32, 16, -5, False), d.DDP_ERR_ARG), ((4097, 32, 16, 128, False), d.DDP_ERR_UNSUPPORTED),
                       ((2, 1025, 16, 128, False), d.DDP_ERR_UNSUPPORTED), ((2, 32, 16, (1 << 20) + 1, False), d.DDP_ERR_UNSUPPORTED)):
        refused(d, code, d.ddp_position_bias_create, d.DDP_DEVICE_NONE, 0, *args)
    for args, code in (((0, 1), d.DDP_ERR_ARG), ((8, 0), d.DDP_ERR_ARG), ((8, 9), d.DDP_ERR_ARG), ((8, 2, 0), d.DDP_ERR_ARG), ((8, 2, 3), d.DDP_ERR_ARG),
                       ((8, 2, 4, 0), d.DDP_ERR_ARG), ((8, 2, 4, 5), d.DDP_ERR_ARG), ((8, 5, 4, 2), d.DDP_ERR_ARG), ((8, 2, 4, 2, 0), d.DDP_ERR_ARG),
                       ((8, 2, 4, 2, 3), d.DDP_ERR_ARG), ((8, 2, 1, 1, 1, 2), d.DDP_ERR_ARG), ((8, 2, 1, 1, 1, 0, True, float("nan")), d.DDP_ERR_ARG),
                       ((8, 2, 1, 1, 1, 0, True, float("inf")), d.DDP_ERR_ARG), ((1025, 2), d.DDP_ERR_UNSUPPORTED), ((128, 65), d.DDP_ERR_UNSUPPORTED),
                       ((130, 2, 65, 65), d.DDP_ERR_UNSUPPORTED)):
        refused(d, code, d.ddp_router_create, d.DDP_DEVICE_NONE, 0, *args)
    for name in ("layernorm", "position_bias", "router"):
        assert getattr(d.binding._lib, f"ddp_{name}_destroy")(None) == d.DDP_ERR_ARG


def test_layernorm_forward(d):
    h = d.ddp_layernorm_create(d.DDP_DEVICE_NONE, 0, 16)
    ok = dict(rows=4, x=256, x_dtype=BF16, x_stride=16, residual=256, residual_stride=16, gamma=256, beta=256, param_dtype=FP32, eps=1e-5, sum_=256,
              sum_stride=16, y=256, y_dtype=BF16, y_stride=16, mean=256, rstd=256)
    f = d.ddp_layernorm_forward
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok))
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, residual=0, residual_stride=0, gamma=0, beta=None, sum_=0, sum_stride=0, mean=0, rstd=0))
    for at in (dict(rows=-1), dict(rows=1 << 31), dict(x_dtype=3), dict(y_dtype=-1), dict(param_dtype=7), dict(eps=-1e-5), dict(eps=float("nan")),
               dict(x_stride=15), dict(y_stride=15), dict(residual_stride=15), dict(sum_stride=0), dict(x_stride=1 << 31), dict(x=0), dict(y=0),
               dict(x=257), dict(y=257), dict(residual=257), dict(sum_=257), dict(gamma=258), dict(beta=257), dict(mean=258), dict(rstd=259)):
        refused(d, d.DDP_ERR_ARG, f, h, *changed(ok, **at))
    for x, y in ((BF16, FP16), (BF16, FP32), (FP16, BF16), (FP16, FP32)):
        refused(d, d.DDP_ERR_UNSUPPORTED, f, h, *changed(ok, x_dtype=x, y_dtype=y))
    assert d.binding._lib.ddp_layernorm_forward(None, *changed(ok)) == d.DDP_ERR_ARG
    with pytest.raises(TypeError):
        f(h, *changed(ok, rows=4.0))
    d.ddp_layernorm_destroy(h)


def test_layernorm_backward(d):
    h = d.ddp_layernorm_create(d.DDP_DEVICE_NONE, 0, 16)
    ok = dict(rows=4, dy=256, dy_dtype=FP16, dy_stride=16, x=256, x_dtype=FP32, x_stride=16, mean=256, rstd=256, gamma=256, param_dtype=FP32, dsum=256,
              dsum_stride=16, dx=256, dx_stride=16, accumulate=True, dgamma=256, dbeta=256, grad_dtype=BF16)
    f = d.ddp_layernorm_backward
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok))
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, gamma=0, dsum=0, dsum_stride=0, dx=0, dx_stride=0, dgamma=0, dbeta=0))
    for at in (dict(rows=-1), dict(rows=1 << 31), dict(x_dtype=3), dict(dy_dtype=-1), dict(param_dtype=7), dict(grad_dtype=3), dict(x_stride=15),
               dict(dy_stride=15), dict(dsum_stride=15), dict(dx_stride=0), dict(dy_stride=1 << 31), dict(x=0), dict(dy=0), dict(mean=0), dict(rstd=0),
               dict(x=258), dict(dy=257), dict(dsum=258), dict(dx=258), dict(gamma=258), dict(mean=258), dict(rstd=259), dict(dgamma=257),
               dict(dbeta=257)):
        refused(d, d.DDP_ERR_ARG, f, h, *changed(ok, **at))
    refused(d, d.DDP_ERR_UNSUPPORTED, f, h, *changed(ok, x_dtype=BF16))
    assert d.binding._lib.ddp_layernorm_backward(None, *changed(ok)) == d.DDP_ERR_ARG
    d.ddp_layernorm_destroy(h)


def test_position_bias_apply(d):
    h = d.ddp_position_bias_create(d.DDP_DEVICE_NONE, 0, 3, 32, 16, 128, False)
    ok = dict(batch=2, queries=5, keys=7, offset=2, table=256, table_dtype=FP32, table_stride=3, scale=1.0, key_lengths=256, causal=True, masked=-1.0,
              accumulate=False, out=256, out_dtype=BF16, batch_stride=105, head_stride=35, query_stride=7)
    f = d.ddp_position_bias_apply
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok))
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, key_lengths=None, masked=float("-inf")))
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, head_stride=7, query_stride=21))            # heads inside a query
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, batch=1, batch_stride=0))
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, batch=0, table=0, out=0))
    for at in (dict(batch=-1), dict(queries=-1), dict(keys=-1), dict(table_dtype=3), dict(out_dtype=-1), dict(table_stride=2), dict(table_stride=1 << 31),
               dict(table=0), dict(out=0), dict(table=258), dict(out=257), dict(key_lengths=258), dict(query_stride=6), dict(head_stride=34),
               dict(batch_stride=104), dict(batch_stride=0), dict(head_stride=-35), dict(query_stride=0), dict(head_stride=7, query_stride=20),
               dict(batch_stride=1 << 47)):
        refused(d, d.DDP_ERR_ARG, f, h, *changed(ok, **at))
    for at in (dict(batch=(1 << 20) + 1), dict(queries=BIG + 1), dict(keys=BIG + 1), dict(offset=BIG + 1), dict(offset=-BIG - 1)):
        refused(d, d.DDP_ERR_UNSUPPORTED, f, h, *changed(ok, **at))
    assert d.binding._lib.ddp_position_bias_apply(None, *changed(ok)) == d.DDP_ERR_ARG
    assert d.binding._lib.ddp_position_bias_buckets(None, None) == d.DDP_ERR_ARG
    assert d.binding._lib.ddp_position_bias_buckets(h, None) == d.DDP_ERR_ARG
    d.ddp_position_bias_destroy(h)


def test_position_bias_grad(d):
    h = d.ddp_position_bias_create(d.DDP_DEVICE_NONE, 0, 3, 32, 16, 128, False)
    ok = dict(batch=2, queries=5, keys=7, offset=2, dscores=256, dtype=BF16, batch_stride=105, head_stride=35, query_stride=7, scale=1.0,
              key_lengths=256, query_lengths=256, causal=True, accumulate=False, grad=256, grad_dtype=FP32, grad_stride=3)
    f = d.ddp_position_bias_grad
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok))
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, key_lengths=0, query_lengths=None, batch_stride=0, head_stride=0, query_stride=0))
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, batch=0, dscores=0))
    for at in (dict(batch=-1), dict(queries=-1), dict(keys=-1), dict(dtype=3), dict(grad_dtype=-1), dict(grad_stride=2), dict(dscores=0), dict(grad=0),
               dict(dscores=257), dict(grad=258), dict(key_lengths=258), dict(query_lengths=257), dict(query_stride=-1), dict(head_stride=-1),
               dict(batch_stride=-1), dict(query_stride=1 << 46), dict(batch_stride=1 << 47)):
        refused(d, d.DDP_ERR_ARG, f, h, *changed(ok, **at))
    for at in (dict(batch=(1 << 20) + 1), dict(queries=BIG + 1), dict(keys=BIG + 1), dict(offset=BIG + 1)):
        refused(d, d.DDP_ERR_UNSUPPORTED, f, h, *changed(ok, **at))
    assert d.binding._lib.ddp_position_bias_grad(None, *changed(ok)) == d.DDP_ERR_ARG
    d.ddp_position_bias_destroy(h)


def test_router(d):
    h = d.ddp_router_create(d.DDP_DEVICE_NONE, 0, 8, 2, 4, 2)
    ok = dict(tokens=3, logits=256, dtype=BF16, stride=8, bias=256, experts_out=256, weights=256, weights_dtype=FP16, counts=256, accumulate=False)
    f = d.ddp_router_route
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok))
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, bias=0, counts=None))
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok, tokens=0, logits=0, experts_out=0, weights=0))
    for at in (dict(tokens=-1), dict(tokens=1 << 31), dict(dtype=3), dict(weights_dtype=-1), dict(stride=7), dict(stride=1 << 31), dict(logits=0),
               dict(experts_out=0), dict(weights=0), dict(logits=257), dict(bias=258), dict(experts_out=258), dict(weights=257), dict(counts=259)):
        refused(d, d.DDP_ERR_ARG, f, h, *changed(ok, **at))
    assert d.binding._lib.ddp_router_route(None, *changed(ok)) == d.DDP_ERR_ARG
    ok = dict(tokens=3, logits=256, dtype=BF16, stride=8, experts_in=256, dweights=256, dweights_dtype=FP16, dlogits=256, dlogits_stride=8)
    f = d.ddp_router_grad
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok))
    for at in (dict(tokens=-1), dict(dtype=3), dict(dweights_dtype=-1), dict(stride=7), dict(dlogits_stride=7), dict(logits=0), dict(experts_in=0),
               dict(dweights=0), dict(dlogits=0), dict(logits=257), dict(experts_in=258), dict(dweights=257), dict(dlogits=257)):
        refused(d, d.DDP_ERR_ARG, f, h, *changed(ok, **at))
    assert d.binding._lib.ddp_router_grad(None, *changed(ok)) == d.DDP_ERR_ARG
    ok = dict(replicas=2, counts=256, rate=1e-3, bias=256, bias_out=256)
    f = d.ddp_router_balance
    refused(d, d.DDP_ERR_NO_DEVICE, f, h, *changed(ok))
    for at in (dict(replicas=0), dict(replicas=d.DDP_MAX_REPLICAS + 1), dict(counts=0), dict(bias=0), dict(bias_out=0), dict(counts=258), dict(bias=258),
               dict(bias_out=257)):
        refused(d, d.DDP_ERR_ARG, f, h, *changed(ok, **at))
    assert d.binding._lib.ddp_router_balance(None, *changed(ok)) == d.DDP_ERR_ARG
    d.ddp_router_destroy(h)


def test_first_distances(d):
    h = d.ddp_position_bias_create(d.DDP_DEVICE_NONE, 0, 1, 8, 4, 64, False)
    assert d.ddp_position_bias_buckets(h).tolist() == [0, 1, 2, 3, 4, 8, 16, 32]
    d.ddp_position_bias_destroy(h)
    h = d.ddp_position_bias_create(d.DDP_DEVICE_NONE, 0, 1, 16, 8, 0, True)
    assert d.ddp_position_bias_buckets(h).tolist() == list(range(8))
    d.ddp_position_bias_destroy(h)
