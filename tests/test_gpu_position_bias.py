"""The relative position bias and its gradient through the C ABI against the 64-bit oracle.

A bias is one binary32 product (and one sum), rounded to the type of the output: compared bit for bit.  A gradient is a sum of n
terms in binary32 along a diagonal and a part of the batch, joined in binary64: its error is at most (n + 16) u times the terms' magnitudes, n the
longest diagonal times the batch, plus one rounding to the gradient's type."""
import numpy as np
import pytest

from layer_cases import BF16, FP16, FP32, GUARD, TINY, U, UNIT, close, lib, torch_type, vector
from oracle import layer as ops

pytestmark = pytest.mark.gpu

KINDS = [(32, 16, 128, False), (32, 8, 128, True), (1, 1, 1, False), (2, 1, 1, True), (6, 3, 0, True), (40, 10, 3000, False), (1024, 256, 5000, True)]
SHAPES = [(1, 1, 1, 1, 0), (2, 3, 5, 9, 0), (1, 2, 1, 300, 299), (2, 2, 70, 33, -40), (1, 1, 130, 515, 385), (3, 2, 64, 64, 0)]


def scores_on(values, dt, gap=0, layout="bhqk", shift=0):
    """values[B, H, Q, K] in a buffer with `gap` further keys a row: (buffer, view)."""
    import torch
    B, H, Q, K = values.shape
    order = {"bhqk": (0, 1, 2), "bqhk": (0, 2, 1), "hbqk": (1, 0, 2)}[layout]
    sizes = [values.shape[i] for i in order]
    buf = torch.full((shift + sizes[0] * sizes[1] * sizes[2] * (K + gap) + 16,), GUARD, dtype=torch_type(dt), device="cuda")
    view = buf[shift:shift + sizes[0] * sizes[1] * sizes[2] * (K + gap)].view(*sizes, K + gap)[..., :K]
    view = view.permute(*[order.index(i) for i in range(3)], 3)
    view.copy_(torch.from_numpy(np.ascontiguousarray(values)))
    return buf, view


def lengths_on(lengths):
    import torch
    return None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")


def ptr(x):
    return 0 if x is None else x.data_ptr()


def check_apply(shape, kind, tt, ot, causal=False, lengths=None, add=False, gap=0, layout="bhqk", shift=0, scale=1.25, masked=-1e9, seed=0,
                stride=0):
    torch, d = lib()
    B, H, Q, K, offset = shape
    rng = np.random.default_rng(seed + Q * 7 + K)
    before = rng.standard_normal((B, H, Q, K))
    seen = ops.visible(B, Q, K, offset, causal, lengths)
    before[~np.broadcast_to(seen[:, None], before.shape)] = np.nan          # what is masked is not used
    buf, out = scores_on(before, ot, gap, layout, shift)
    held = out.float().cpu().numpy()
    table, _ = vector(rng.standard_normal((kind[0], H + stride)), tt)
    on = lengths_on(lengths)
    h = d.ddp_position_bias_create(0, 0, H, *kind)
    torch.cuda.synchronize()
    d.ddp_position_bias_apply(h, B, Q, K, offset, table.data_ptr(), tt, H + stride, scale, ptr(on), causal, masked, add, out.data_ptr(), ot,
                              out.stride(0), out.stride(1), out.stride(2))
    torch.cuda.synchronize()
    places = ops.bucket_places(Q, K, offset, *kind)
    want = (table.float().cpu().numpy()[places][:, :, :H] * np.float32(scale)).transpose(2, 0, 1)[None]
    want = held + want if add else np.broadcast_to(want, held.shape)
    want = np.where(seen[:, None], want, np.float32(masked))
    assert want.dtype == np.float32
    want = torch.from_numpy(np.ascontiguousarray(want)).to(torch_type(ot))
    got = out.cpu()
    assert torch.equal(got, want), np.argwhere((got != want).numpy())[:4].tolist()
    out.fill_(GUARD)
    assert (buf == GUARD).all(), "wrote outside its rows"
    d.ddp_position_bias_destroy(h)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
def test_apply(shape, kind):
    check_apply(shape, kind, FP32, BF16)
    check_apply(shape, kind, BF16, FP32, causal=True)


@pytest.mark.parametrize("tt", [FP32, FP16, BF16])
@pytest.mark.parametrize("ot", [FP32, FP16, BF16])
@pytest.mark.parametrize("add", [False, True])
def test_apply_types(tt, ot, add):
    check_apply((2, 3, 37, 75, 3), (32, 8, 128, True), tt, ot, causal=True, add=add, masked=-6e4)


@pytest.mark.parametrize("layout", ["bhqk", "bqhk", "hbqk"])
@pytest.mark.parametrize("gap,shift,stride", [(0, 0, 0), (3, 1, 2), (8, 8, 0), (0, 5, 1)])
@pytest.mark.parametrize("ot", [FP32, BF16])
def test_apply_strides(layout, gap, shift, stride, ot):
    check_apply((2, 3, 41, 66, 0), (32, 16, 128, False), FP32, ot, add=True, gap=gap, layout=layout, shift=shift, stride=stride)


@pytest.mark.parametrize("lengths", [[0, 1, 50], [50, 49, -3], [77, 25, 8]])
@pytest.mark.parametrize("causal,masked", [(False, -np.inf), (True, -np.inf), (True, float(np.finfo(np.float32).min))])
def test_apply_lengths(lengths, causal, masked):
    check_apply((3, 2, 20, 50, 10), (32, 16, 128, False), FP32, FP32, causal=causal, lengths=lengths, masked=masked)
    check_apply((3, 2, 20, 50, 10), (32, 16, 128, False), FP32, FP16, causal=causal, lengths=lengths, add=True, masked=masked if np.isinf(masked) else -65504.0)


def test_apply_with_rows_that_see_nothing():
    check_apply((1, 2, 40, 30, -25), (32, 16, 128, False), FP32, BF16, causal=True, masked=-np.inf)


@pytest.mark.parametrize("keys", [1, 7, 8, 9, 511, 512, 513, 2047, 4097])
def test_apply_for_a_single_token(keys):
    check_apply((2, 3, 1, keys, keys - 1), (32, 16, 128, False), FP32, BF16, causal=True)
    check_apply((1, 3, 1, keys, keys - 1), (32, 16, 128, False), BF16, FP32, gap=1, add=True)


@pytest.mark.parametrize("queries,keys,offset", [(700, 520, 0), (259, 1100, 841), (1030, 90, -500)])
@pytest.mark.parametrize("ot", [FP32, BF16])
def test_apply_of_longer_scores(queries, keys, offset, ot):
    check_apply((1, 2, queries, keys, offset), (32, 16, 500, False), FP32, ot, causal=True)
    check_apply((2, 1, queries, keys, offset), (64, 9, 300, True), FP32, ot, lengths=[keys, keys // 2], add=True)


def test_buckets_of_the_handle_are_those_of_the_oracle():
    _, d = lib()
    for kind in KINDS + [(512, 16, 1 << 20, False), (30, 2, 2 << 13, True), (17, 1, 1 << 16, False)]:
        h = d.ddp_position_bias_create(d.DDP_DEVICE_NONE, 0, 1, *kind)
        first = d.ddp_position_bias_buckets(h)
        n = kind[0] // 2 if kind[3] else kind[0]
        assert len(first) == n
        for k, at in enumerate(first):
            for r in {max(int(at) - 1, 0), int(at), int(at) + 1}:
                assert np.searchsorted(first, r, side="right") - 1 == ops.bucket(-r, *kind), (kind, k, r)
        d.ddp_position_bias_destroy(h)


def check_grad(shape, kind, st, gt, causal=False, key_lengths=None, query_lengths=None, add=False, gap=0, layout="bhqk", shift=0, scale=1.25, seed=0,
               stride=0, handle=None, values=None):
    torch, d = lib()
    B, H, Q, K, offset = shape
    rng = np.random.default_rng(seed + Q * 5 + K)
    ds = rng.standard_normal((B, H, Q, K)) if values is None else values
    seen = ops.visible(B, Q, K, offset, causal, key_lengths, query_lengths)
    ds[~np.broadcast_to(seen[:, None], ds.shape)] = np.nan                  # what is masked is not used
    buf, on = scores_on(ds, st, gap, layout, shift)
    held = np.nan_to_num(on.double().cpu().numpy())
    grad, old = vector(rng.standard_normal((kind[0], H + stride)), gt)
    before = grad.clone()
    kl, ql = lengths_on(key_lengths), lengths_on(query_lengths)
    h = handle or d.ddp_position_bias_create(0, 0, H, *kind)
    torch.cuda.synchronize()
    d.ddp_position_bias_grad(h, B, Q, K, offset, on.data_ptr(), st, on.stride(0), on.stride(1), on.stride(2), scale, ptr(kl), ptr(ql), causal, add,
                             grad.data_ptr(), gt, H + stride)
    torch.cuda.synchronize()
    want, magnitude = ops.bias_grad(held, seen, ops.bucket_places(Q, K, offset, *kind), kind[0])
    want, magnitude = scale * want, scale * magnitude
    if add:
        want, magnitude = want + old[:, :H], magnitude + np.abs(old[:, :H])
    bound = (min(Q, K) * B + 16) * U * magnitude + UNIT[gt] * np.abs(want) + TINY[gt]
    close(grad[:, :H].double().cpu().numpy(), want, bound, "grad")
    assert torch.equal(grad[:, H:], before[:, H:])
    if handle is None:
        d.ddp_position_bias_destroy(h)
    return grad


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
def test_grad(shape, kind):
    check_grad(shape, kind, FP32, FP32)
    check_grad(shape, kind, BF16, FP32, causal=True, add=True)


@pytest.mark.parametrize("st", [FP32, FP16, BF16])
@pytest.mark.parametrize("gt", [FP32, FP16, BF16])
@pytest.mark.parametrize("add", [False, True])
def test_grad_types(st, gt, add):
    check_grad((2, 3, 37, 75, 3), (32, 8, 128, True), st, gt, causal=True, add=add)


@pytest.mark.parametrize("layout", ["bhqk", "bqhk", "hbqk"])
@pytest.mark.parametrize("gap,shift,stride", [(0, 0, 0), (3, 1, 2), (8, 8, 0), (0, 5, 1)])
@pytest.mark.parametrize("st", [FP32, BF16])
def test_grad_strides(layout, gap, shift, stride, st):
    check_grad((2, 3, 41, 66, 0), (32, 16, 128, False), st, FP32, gap=gap, layout=layout, shift=shift, stride=stride)


@pytest.mark.parametrize("key_lengths", [None, [0, 1, 50], [50, 49, -3], [77, 25, 8]])
@pytest.mark.parametrize("query_lengths", [None, [0, 20, 3], [99, -1, 19]])
@pytest.mark.parametrize("causal", [False, True])
def test_grad_lengths(key_lengths, query_lengths, causal):
    for st in (FP32, BF16):
        check_grad((3, 2, 20, 50, 10), (32, 8, 128, True), st, FP32, causal=causal, key_lengths=key_lengths, query_lengths=query_lengths)


@pytest.mark.parametrize("queries,keys,offset", [(700, 520, 0), (259, 1100, 841), (1030, 90, -500), (1, 4097, 4096), (4097, 1, 0), (2, 2, 5000), (2, 2, -5000)])
@pytest.mark.parametrize("st", [FP32, BF16])
def test_grad_of_longer_scores(queries, keys, offset, st):
    check_grad((1, 2, queries, keys, offset), (32, 16, 500, False), st, FP32, causal=True)
    check_grad((2, 1, queries, keys, offset), (64, 9, 300, True), st, FP32, key_lengths=[keys, keys // 2], query_lengths=[queries // 3, queries])


def test_grad_of_expanded_scores():
    """Strides of 0: the same scores for every sequence and head."""
    torch, d = lib()
    B, H, Q, K, kind = 3, 2, 30, 45, (32, 16, 128, False)
    ds = torch.randn((Q, K), generator=torch.Generator().manual_seed(3)).cuda()
    h = d.ddp_position_bias_create(0, 0, H, *kind)
    grad = torch.zeros((32, H), device="cuda")
    torch.cuda.synchronize()
    d.ddp_position_bias_grad(h, B, Q, K, 0, ds.data_ptr(), FP32, 0, 0, K, 1.0, 0, 0, False, False, grad.data_ptr(), FP32, H)
    torch.cuda.synchronize()
    full = ds.double().cpu().numpy()[None, None].repeat(B, 0).repeat(H, 1)
    want, magnitude = ops.bias_grad(full, ops.visible(B, Q, K, 0), ops.bucket_places(Q, K, 0, *kind), 32)
    close(grad.double().cpu().numpy(), want, (Q * B + 17) * U * magnitude + U * np.abs(want) + 1e-45, "grad")
    d.ddp_position_bias_destroy(h)


def test_grad_of_nothing():
    torch, d = lib()
    h = d.ddp_position_bias_create(0, 0, 3, 32, 16, 128, False)
    grad = torch.full((32, 3), GUARD, device="cuda")
    torch.cuda.synchronize()
    for add, left in ((True, GUARD), (False, 0.0)):
        d.ddp_position_bias_grad(h, 0, 5, 5, 0, 0, FP32, 75, 25, 5, 1.0, 0, 0, False, add, grad.data_ptr(), FP32, 3)
        torch.cuda.synchronize()
        assert (grad == left).all()
    d.ddp_position_bias_apply(h, 1, 0, 5, 0, 0, FP32, 3, 1.0, 0, False, 0.0, False, 0, FP32, 25, 25, 5)
    d.ddp_position_bias_destroy(h)


def test_same_bits_again():
    torch, d = lib()
    kind = (32, 8, 128, True)
    h = d.ddp_position_bias_create(0, 0, 2, *kind)
    first = check_grad((2, 2, 600, 700, 0), kind, BF16, FP32, handle=h)
    check_grad((1, 2, 50, 70, 0), kind, FP32, FP32, handle=h)
    assert torch.equal(first, check_grad((2, 2, 600, 700, 0), kind, BF16, FP32, handle=h))
    d.ddp_position_bias_destroy(h)


def test_scores_past_32_bits():
    """Scores of 5 GB: offsets of the last heads need more than 32 bits.  Ones: a bucket's gradient is the number of its places."""
    torch, d = lib()
    H, Q, K = 40, 8000, 8000
    s = torch.ones((1, H, Q, K), dtype=torch.bfloat16, device="cuda")
    table = torch.arange(4 * H, dtype=torch.float32, device="cuda").view(4, H) % 100
    grad = torch.zeros((4, H), device="cuda")
    h = d.ddp_position_bias_create(0, 0, H, 4, 4, 0, False)
    torch.cuda.synchronize()
    d.ddp_position_bias_grad(h, 1, Q, K, 0, s.data_ptr(), BF16, s.stride(0), s.stride(1), s.stride(2), 1.0, 0, 0, True, False, grad.data_ptr(), FP32, H)
    d.ddp_position_bias_apply(h, 1, Q, K, 0, table.data_ptr(), FP32, H, 1.0, 0, True, -1.0, False, s.data_ptr(), BF16, s.stride(0), s.stride(1),
                              s.stride(2))
    torch.cuda.synchronize()
    far = sum(Q - x for x in range(3, Q))
    want = torch.tensor([Q, Q - 1, Q - 2, far], dtype=torch.float64)
    assert torch.equal(grad.cpu().double(), want.float().double()[:, None].expand(4, H))
    for i in (0, 1, 2, 3, 4000, Q - 1):
        row = s[0, -1, i].float()
        assert (row[i + 1:] == -1.0).all()
        for x in range(0, min(i, 5) + 1):
            assert row[i - x] == table[min(x, 3), -1]
        assert (row[:max(0, i - 2)] == table[3, -1]).all()
    d.ddp_position_bias_destroy(h)


def test_on_another_stream_and_replayed():
    torch, d = lib()
    B, H, Q, K, kind = 2, 4, 300, 300, (32, 16, 128, False)
    stream = torch.cuda.Stream()
    h = d.ddp_position_bias_create(0, stream.cuda_stream, H, *kind)
    table, grad = torch.randn((32, H), device="cuda"), torch.zeros((32, H), device="cuda")
    s = torch.zeros((B, H, Q, K), dtype=torch.bfloat16, device="cuda")
    lengths = torch.tensor([300, 170], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()

    def both():
        d.ddp_position_bias_apply(h, B, Q, K, 0, table.data_ptr(), FP32, H, 1.0, lengths.data_ptr(), True, 0.0, False, s.data_ptr(), BF16, *s.stride()[:3])
        d.ddp_position_bias_grad(h, B, Q, K, 0, s.data_ptr(), BF16, *s.stride()[:3], 1.0, lengths.data_ptr(), 0, True, False, grad.data_ptr(), FP32, H)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        both()
        stream.synchronize()
        graph.capture_begin()
        both()
        graph.capture_end()
        for seed in range(4):
            table.copy_(torch.randn((32, H), generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
            lengths[1] = 10 + 60 * seed
            both()
            stream.synchronize()
            want = s.clone(), grad.clone()
            s.fill_(GUARD)
            grad.fill_(GUARD)
            graph.replay()
            stream.synchronize()
            assert torch.equal(s, want[0]) and torch.equal(grad, want[1])
    torch.cuda.synchronize()
    d.ddp_position_bias_destroy(h)


@pytest.mark.parametrize("batch,queries,keys,offset,causal", [(1, 5000, 5000, 0, True), (2, 3001, 2999, 0, False), (3, 300, 4100, 3800, True), (70, 64, 64, 0, True),
                                                              (2, 4100, 17, -4083, True), (1, 20000, 600, 0, False)])
@pytest.mark.parametrize("dt", [FP32, BF16])
def test_grad_of_small_whole_numbers(batch, queries, keys, offset, causal, dt):
    """Sums of whole numbers are exact at every size: all the ways that strips and row groups are dealt out count every place once."""
    torch, d = lib()
    H, kind = 2, (32, 8, 700, True)
    gen = torch.Generator("cuda").manual_seed(queries)
    ds = torch.randint(-1, 2, (batch, H, queries, keys), generator=gen, device="cuda").to(torch_type(dt))
    lengths = torch.randint(0, queries + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    grad = torch.full((32, H), GUARD, device="cuda")
    h = d.ddp_position_bias_create(0, 0, H, *kind)
    first = torch.from_numpy(d.ddp_position_bias_buckets(h)).cuda().long()
    torch.cuda.synchronize()
    d.ddp_position_bias_grad(h, batch, queries, keys, offset, ds.data_ptr(), dt, *ds.stride()[:3], 1.0, 0, lengths.data_ptr(), causal, False, grad.data_ptr(),
                             FP32, H)
    torch.cuda.synchronize()
    i, j = torch.arange(queries, device="cuda")[:, None], torch.arange(keys, device="cuda")[None]
    r = j - i - offset
    bucket = torch.bucketize(r.abs(), first, right=True) - 1 + (r > 0) * 16
    want = torch.zeros((32, H), device="cuda", dtype=torch.float64)
    for b in range(batch):
        seen = i < lengths[b]
        if causal:
            seen = seen & (r <= 0)
        for n in range(H):
            want[:, n] += torch.bincount(bucket[seen.expand_as(r)], weights=ds[b, n][seen.expand_as(r)].double(), minlength=32)
    assert torch.equal(grad.double(), want)
    d.ddp_position_bias_destroy(h)


@pytest.mark.parametrize("queries,keys,gap,shift", [(1, 1, 0, 3), (9, 3, 0, 1), (40, 61, 0, 5), (7, 64, 0, 0), (64, 7, 1, 2)])
@pytest.mark.parametrize("dt", [FP32, BF16])
def test_grad_at_the_end_of_its_memory(queries, keys, gap, shift, dt):
    """Scores that end with their allocation: nothing behind it is read (what would be is NaN here, and would show)."""
    torch, d = lib()
    B, H, kind = 2, 3, (8, 4, 32, False)
    n = B * H * queries * (keys + gap) - gap
    mem = torch.full((shift + n + 64,), float("nan"), dtype=torch_type(dt), device="cuda")
    view = mem[shift:shift + n].as_strided((B, H, queries, keys), (H * queries * (keys + gap), queries * (keys + gap), keys + gap, 1))
    view.copy_(torch.randint(-3, 4, (B, H, queries, keys), generator=torch.Generator("cuda").manual_seed(keys), device="cuda"))
    grad = torch.zeros((8, H), device="cuda")
    h = d.ddp_position_bias_create(0, 0, H, *kind)
    torch.cuda.synchronize()
    d.ddp_position_bias_grad(h, B, queries, keys, 0, view.data_ptr(), dt, *view.stride()[:3], 1.0, 0, 0, False, False, grad.data_ptr(), FP32, H)
    torch.cuda.synchronize()
    want, _ = ops.bias_grad(view.double().cpu().numpy(), ops.visible(B, queries, keys, 0), ops.bucket_places(queries, keys, 0, *kind), 8)
    assert (grad.double().cpu().numpy() == want).all()
    d.ddp_position_bias_destroy(h)


def test_strides_of_single_entries_may_be_anything():
    torch, d = lib()
    K, kind = 37, (32, 16, 128, False)
    h = d.ddp_position_bias_create(0, 0, 1, *kind)
    table = torch.randn((32, 1), device="cuda")
    out, grad = torch.zeros(K, device="cuda"), torch.zeros((32, 1), device="cuda")
    far = 1 << 62
    torch.cuda.synchronize()
    d.ddp_position_bias_apply(h, 1, 1, K, K - 1, table.data_ptr(), FP32, 1, 1.0, 0, True, 0.0, False, out.data_ptr(), FP32, far, -far, far + 1)
    out_of = out.cpu()
    d.ddp_position_bias_grad(h, 1, 1, K, K - 1, out.data_ptr(), FP32, far, far, far, 1.0, 0, 0, True, False, grad.data_ptr(), FP32, 1)
    torch.cuda.synchronize()
    places = ops.bucket_places(1, K, K - 1, *kind)[0]
    assert torch.equal(out_of, table[:, 0].cpu()[places])
    want = np.bincount(places, weights=out_of.double().numpy(), minlength=32)
    assert np.allclose(grad[:, 0].double().cpu().numpy(), want, rtol=1e-6, atol=1e-6)
    d.ddp_position_bias_destroy(h)


@pytest.mark.parametrize("heads,queries,keys,offset,gap,dt", [(5, 4099, 3331, 0, 0, FP32), (3, 6007, 8009, 2002, 3, BF16)])
def test_apply_beyond_the_caches(heads, queries, keys, offset, gap, dt):
    """More than 256 MiB, tiles of no multiple of eight: every place is written, and none between the rows."""
    torch, d = lib()
    kind = (32, 8, 700, True)
    out = torch.full((heads, queries, keys + gap), GUARD, dtype=torch_type(dt), device="cuda")
    table = torch.randn((32, heads), generator=torch.Generator("cuda").manual_seed(keys), device="cuda")
    h = d.ddp_position_bias_create(0, 0, heads, *kind)
    first = torch.from_numpy(d.ddp_position_bias_buckets(h)).cuda().long()
    torch.cuda.synchronize()
    d.ddp_position_bias_apply(h, 1, queries, keys, offset, table.data_ptr(), FP32, heads, 0.5, 0, True, -7.0, False, out.data_ptr(), dt, 0,
                              out.stride(0), out.stride(1))
    torch.cuda.synchronize()
    r = torch.arange(keys, device="cuda")[None] - torch.arange(queries, device="cuda")[:, None] - offset
    bucket = torch.bucketize(r.abs(), first, right=True) - 1 + (r > 0) * 16
    for n in range(heads):
        want = torch.where(r > 0, torch.full((), -7.0, device="cuda"), (table[:, n] * 0.5)[bucket]).to(out.dtype)
        assert torch.equal(out[n, :, :keys], want)
    assert (out[:, :, keys:] == GUARD).all()
    d.ddp_position_bias_destroy(h)
