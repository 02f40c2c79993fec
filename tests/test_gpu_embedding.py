"""The embedding lookup and its gradient, through the C ABI, against the 64-bit oracle.

A lookup is one binary32 product, rounded to the type of the output: compared bit for bit.  A row of the
gradient is a binary32 sum of n terms, scaled (and added to what is there): its error is at most (n + 3) u times the
sum of the terms' magnitudes, u = 2^-24, plus one rounding to the gradient's type."""
import numpy as np
import pytest

from oracle import operators as ops

pytestmark = pytest.mark.gpu

FP32, FP16, BF16 = 0, 1, 2
U = 2.0 ** -24
UNIT = {FP32: 0.0, FP16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {FP32: 2.0 ** -149, FP16: 2.0 ** -25, BF16: 2.0 ** -134}


def lib():
    import torch
    import paper_2006_15704_amd as d
    return torch, d


def torch_type(torch, dt):
    return {FP32: torch.float32, FP16: torch.float16, BF16: torch.bfloat16}[dt]


def rows_of(values, dt, stride, shift=0, guard=7.0):
    """values[T, D] in a buffer with `stride` elements from row to row, `shift` elements in: (buffer, view)."""
    torch, _ = lib()
    T, D = values.shape
    buf = torch.full((shift + T * stride + 16,), guard, dtype=torch_type(torch, dt), device="cuda")
    view = buf[shift:shift + T * stride].view(T, stride)[:, :D]
    view.copy_(torch.from_numpy(np.ascontiguousarray(values, dtype=np.float64)))
    return buf, view


def ids_on(ids, bits, shift=0):
    torch, _ = lib()
    buf = torch.zeros(len(ids) + shift, dtype=torch.int64 if bits == 64 else torch.int32, device="cuda")
    buf[shift:].copy_(torch.from_numpy(np.asarray(ids, dtype=np.int64)))
    return buf[shift:]


def check_lookup(rows, width, ids, table_dt, out_dt, bits=64, gaps=(0, 0), shifts=(0, 0), scale=1.5, seed=0):
    torch, d = lib()
    rng = np.random.default_rng(seed)
    T = len(ids)
    _, table = rows_of(rng.standard_normal((rows, width)), table_dt, width + gaps[0], shifts[0])
    out_buf, out = rows_of(np.full((T, width), 7.0), out_dt, width + gaps[1], shifts[1])
    on = ids_on(ids, bits)
    emb = d.ddp_embedding_create(0, 0, rows, width, 0)
    torch.cuda.synchronize()
    d.ddp_embedding_lookup(emb, T, on.data_ptr(), bits, table.data_ptr(), table_dt, width + gaps[0], scale, out.data_ptr(),
                           out_dt, width + gaps[1])
    torch.cuda.synchronize()
    held = table.double().cpu().numpy()
    want = torch.from_numpy(ops.lookup(held, np.asarray(ids), np.float32(scale)).astype(np.float32)).to(torch_type(torch, out_dt))
    assert torch.equal(out.cpu(), want)
    keep = out_buf.clone()
    keep[shifts[1]:shifts[1] + T * (width + gaps[1])].view(T, width + gaps[1])[:, :width] = 7.0
    assert (keep == 7.0).all(), "wrote outside its rows"
    d.ddp_embedding_destroy(emb)


@pytest.mark.parametrize("table_dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("out_dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("width,tokens", [(1, 1), (7, 5), (64, 3), (513, 9), (1024, 1), (2050, 6)])
def test_lookup(table_dt, out_dt, width, tokens):
    rng = np.random.default_rng(width)
    check_lookup(37, width, rng.integers(0, 37, tokens), table_dt, out_dt)


@pytest.mark.parametrize("bits", [32, 64])
def test_lookup_outside_the_table(bits):
    far = 2 ** 31 - 1 if bits == 32 else 2 ** 40
    check_lookup(5, 100, [0, -1, 4, 5, far, -far, 2], FP32, BF16, bits)


@pytest.mark.parametrize("gaps,shifts", [((3, 0), (0, 1)), ((0, 5), (1, 3)), ((1, 1), (1, 0)), ((8, 8), (4, 4))])
@pytest.mark.parametrize("dt", [FP32, BF16])
def test_lookup_strides_and_alignments(gaps, shifts, dt):
    check_lookup(19, 130, np.arange(40) % 19, dt, dt, gaps=gaps, shifts=shifts)


def test_lookup_past_32_bits():
    """A table of 4.3 GB: the offset of its last rows needs more than 32 bits."""
    torch, d = lib()
    rows, width = 1 << 21, 1040
    table = torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda")
    table[-1], table[rows // 2 + 1] = 3.0, 5.0
    ids = ids_on([rows - 1, rows // 2 + 1, 0], 64)
    out = torch.full((3, width), 7.0, device="cuda")
    emb = d.ddp_embedding_create(0, 0, rows, width, 0)
    torch.cuda.synchronize()
    d.ddp_embedding_lookup(emb, 3, ids.data_ptr(), 64, table.data_ptr(), BF16, width, 2.0, out.data_ptr(), FP32, width)
    torch.cuda.synchronize()
    assert (out[0] == 6.0).all() and (out[1] == 10.0).all() and (out[2] == 0.0).all()
    d.ddp_embedding_destroy(emb)


class Table:
    def __init__(self, rows, width, max_tokens, stream=0):
        _, d = lib()
        self.rows, self.width = rows, width
        self.emb = d.ddp_embedding_create(0, stream, rows, width, max_tokens)

    def grad(self, ids, dout, dout_dt, grad, grad_dt, scale=1.5, padding=-1, add=False, bits=64, gaps=(0, 0)):
        _, d = lib()
        d.ddp_embedding_grad(self.emb, len(ids), ids.data_ptr(), bits, dout.data_ptr(), dout_dt, self.width + gaps[0], scale,
                             padding, add, grad.data_ptr(), grad_dt, self.width + gaps[1])

    def close(self):
        _, d = lib()
        d.ddp_embedding_destroy(self.emb)


def check_grad(rows, width, ids, dout_dt, grad_dt, padding=-1, add=False, bits=64, gaps=(0, 0), shifts=(0, 0), seed=0, table=None,
               poison=False, scale=1.5):
    torch, _ = lib()
    rng = np.random.default_rng(seed)
    ids = np.asarray(ids, dtype=np.int64)
    T = len(ids)
    unused = (ids < 0) | (ids >= rows) | (ids == padding)
    _, dout = rows_of(rng.standard_normal((T, width)) if T else np.zeros((0, width)), dout_dt, width + gaps[0], shifts[0])
    if poison:
        dout[torch.from_numpy(unused).cuda()] = float("nan")
    buf, grad = rows_of(rng.standard_normal((rows, width)), grad_dt, width + gaps[1], shifts[1])
    if poison and not add:
        grad.fill_(float("nan"))
    old = grad.double().cpu().numpy() if add else None
    mine = table or Table(rows, width, max(T, 1))
    on = ids_on(ids, bits)
    torch.cuda.synchronize()
    mine.grad(on, dout, dout_dt, grad, grad_dt, scale, padding, add, bits, gaps)
    torch.cuda.synchronize()
    held = np.nan_to_num(dout.double().cpu().numpy())
    want, size = ops.embedding_grad(rows, ids, held, float(np.float32(scale)), padding, old)
    count = np.bincount(ids[~unused], minlength=rows)[:, None]
    got = grad.double().cpu().numpy()
    assert (np.abs(got - want) <= (count + 3) * U * size + UNIT[grad_dt] * np.abs(want) + TINY[grad_dt]).all()
    if add:
        assert (got[count[:, 0] == 0] == old[count[:, 0] == 0]).all(), "a row without tokens was touched"
    keep = buf.clone()
    keep[shifts[1]:shifts[1] + rows * (width + gaps[1])].view(rows, width + gaps[1])[:, :width] = 7.0
    assert (keep == 7.0).all(), "wrote outside its rows"
    if table is None:
        mine.close()
    return got


def zipf(rng, rows, tokens):
    return np.minimum(np.exp(rng.random(tokens) * np.log(rows + 1.0)).astype(np.int64) - 1, rows - 1)


@pytest.mark.parametrize("dout_dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("grad_dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("add", [False, True])
def test_grad_types(dout_dt, grad_dt, add):
    rng = np.random.default_rng(1)
    check_grad(50, 130, zipf(rng, 50, 333), dout_dt, grad_dt, add=add)


@pytest.mark.parametrize("rows,width,tokens", [
    (1, 1, 1), (1, 5, 1000), (2, 64, 512), (3, 1024, 2), (16, 8, 17), (17, 520, 33), (1000, 3, 1023), (1024, 16, 1024),
    (1025, 16, 1025), (2049, 4, 5000), (5000, 40, 100), (40000, 12, 20000), (513, 1030, 600), (70000, 130, 1500),
    (30001, 30, 4096), (600, 2000, 3000)])
@pytest.mark.parametrize("spread", ["zipf", "even", "one"])
def test_grad_sizes(rows, width, tokens, spread):
    rng = np.random.default_rng(rows + tokens)
    ids = zipf(rng, rows, tokens) if spread == "zipf" else rng.integers(0, rows, tokens) if spread == "even" else np.full(tokens, rows - 1)
    check_grad(rows, width, ids, BF16, FP32)


@pytest.mark.parametrize("rows,tokens", [(1 << 20, 5000), ((1 << 20) + 3, 9000), (70000, 30000)])
def test_grad_many_rows(rows, tokens):
    """Buckets of up to 1024 rows, more than 1024 buckets; spread thin, and with frequent rows."""
    rng = np.random.default_rng(rows)
    check_grad(rows, 4, rng.integers(0, rows, tokens), BF16, FP32)
    check_grad(rows, 4, zipf(rng, rows, tokens), FP32, FP32, add=True)
    check_grad(rows, 4, rng.integers(0, 3, tokens) * 1024 + rng.integers(0, 2, tokens), FP16, FP32)


@pytest.mark.parametrize("tokens", [0, 1, 31, 32, 33, 63, 64, 65, 96, 97, 4095, 4096, 4097])
def test_grad_of_one_row(tokens):
    """Every length at which a row's tokens are split or end a part, next to rows with one token."""
    ids = np.concatenate([[0], np.full(tokens, 1), [3]])
    check_grad(5, 20, ids, FP32, FP32)


@pytest.mark.parametrize("lengths", [(33, 33, 33), (40, 1, 40), (32, 33, 31, 64), (1, 100, 1, 100), (33, 31, 33, 31, 1)])
def test_grad_rows_that_meet_in_a_window(lengths):
    ids = np.concatenate([np.full(n, r) for r, n in enumerate(lengths)])
    for seed in range(2):
        check_grad(len(lengths), 24, np.random.default_rng(seed).permutation(ids), BF16, BF16, seed=seed)


@pytest.mark.parametrize("padding", [-1, 0, 6])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("bits", [32, 64])
def test_grad_padding_is_not_read(padding, add, bits):
    """Rows of dout whose token takes no part hold NaN, and so does the gradient that is overwritten."""
    rng = np.random.default_rng(3)
    ids = rng.integers(-3, 12, 500)
    ids[7], ids[8] = (2 ** 31 - 1, -2 ** 31) if bits == 32 else (2 ** 40, -2 ** 50)
    check_grad(9, 77, ids, BF16, FP32, padding=padding, add=add, bits=bits, poison=True)


def test_grad_without_a_token_that_counts():
    got = check_grad(9, 33, np.full(700, 4), FP32, FP16, padding=4, poison=True)
    assert (got == 0).all()
    check_grad(9, 33, np.full(700, -1), FP32, FP16, add=True)
    check_grad(9, 33, [], FP32, FP16, poison=True)
    check_grad(9, 33, [], FP32, FP16, add=True)


@pytest.mark.parametrize("gaps,shifts", [((3, 0), (0, 1)), ((0, 5), (1, 3)), ((1, 1), (1, 0)), ((8, 8), (4, 4))])
@pytest.mark.parametrize("dt", [FP32, FP16])
def test_grad_strides_and_alignments(gaps, shifts, dt):
    rng = np.random.default_rng(4)
    check_grad(61, 131, zipf(rng, 61, 400), dt, dt, gaps=gaps, shifts=shifts)
    check_grad(61, 131, zipf(rng, 61, 400), dt, dt, gaps=gaps, shifts=shifts, add=True)


@pytest.mark.parametrize("tokens", [9, 1500])
def test_grad_past_32_bits(tokens):
    """Rows of dout and of the gradient whose offsets need more than 32 bits, by either way through the tokens."""
    torch, d = lib()
    rows, width, dout_stride, grad_stride = 5, 1040, (1 << 32) // tokens, 1 << 30
    ids = np.arange(tokens) % (rows - 1) + 1
    dout = torch.empty(tokens * dout_stride + width, dtype=torch.bfloat16, device="cuda")[:tokens * dout_stride].view(tokens, dout_stride)
    grad = torch.empty(rows * grad_stride, dtype=torch.bfloat16, device="cuda").view(rows, grad_stride)
    dout[:, :width] = torch.arange(tokens, device="cuda").remainder(7).bfloat16()[:, None]
    grad[:, :width + 8] = 7.0
    on, emb = ids_on(ids, 64), d.ddp_embedding_create(0, 0, rows, width, tokens)
    torch.cuda.synchronize()
    d.ddp_embedding_grad(emb, tokens, on.data_ptr(), 64, dout.data_ptr(), BF16, dout_stride, 0.5, -1, False, grad.data_ptr(), BF16, grad_stride)
    torch.cuda.synchronize()
    got = grad[:, :width + 8].double().cpu().numpy()
    want = 0.5 * np.bincount(ids, weights=np.arange(tokens) % 7, minlength=rows)[:, None]
    assert (np.abs(got[:, :width] - want) <= UNIT[BF16] * want).all() and (got[:, width:] == 7.0).all()
    d.ddp_embedding_destroy(emb)


def test_grad_values_that_are_not_finite_stay_in_their_row():
    torch, _ = lib()
    dout = torch.ones((40, 16), device="cuda")
    dout[3, 5], dout[9, 2] = float("inf"), float("nan")
    grad = torch.empty((6, 16), device="cuda")
    ids = ids_on([i % 4 for i in range(40)], 64)
    t = Table(6, 16, 40)
    t.grad(ids, dout, FP32, grad, FP32, 1.0)
    torch.cuda.synchronize()
    bad = (~torch.isfinite(grad)).nonzero().cpu().tolist()
    assert bad == [[1, 2], [3, 5]]
    t.close()


@pytest.mark.parametrize("tokens", [4097, 9000, 40000])
def test_grad_long_calls_of_few_rows(tokens):
    """Every row is split into many parts; a bucket holds more tokens than LDS does."""
    rng = np.random.default_rng(tokens)
    check_grad(2, 260, rng.integers(0, 2, tokens), FP32, FP32)
    check_grad(1, 8, np.zeros(tokens), BF16, BF16)
    check_grad(40, 12, zipf(rng, 40, tokens), BF16, FP32, padding=0, poison=True)
    check_grad(3000, 9, np.where(rng.random(tokens) < 0.7, 1024, rng.integers(0, 3000, tokens)), FP16, FP32)


@pytest.mark.parametrize("rows", [2, 33, 120])
def test_grad_long_windows(rows):
    """Tables of few and wide rows have longer parts: rows of more, fewer and just as many tokens."""
    rng = np.random.default_rng(rows)
    ids = zipf(rng, rows, 40000)
    if rows > 100:
        for r, n in ((100, 127), (101, 128), (102, 129), (103, 64), (104, 65), (105, 1)):
            ids[ids == r] = 0
            ids[rng.choice(np.flatnonzero(ids == 0), n, replace=False)] = r
    check_grad(rows, 1030, ids, FP32, FP32)
    check_grad(rows, 2060, ids, BF16, BF16, add=True)


def test_grad_calls_do_not_see_each_other():
    """One handle, calls of different lengths and spreads in turn: nothing of a longer call is left."""
    rng = np.random.default_rng(5)
    t = Table(3000, 48, 30000)
    for k, tokens in enumerate((30000, 10, 0, 5000, 1, 29999, 1024)):
        ids = zipf(rng, 3000, tokens) if k % 2 else rng.integers(-5, 3000, tokens)
        check_grad(3000, 48, ids, BF16, FP32, seed=k, table=t)
    t.close()


def test_grad_same_bits_every_time():
    torch, _ = lib()
    rng = np.random.default_rng(6)
    ids = ids_on(zipf(rng, 2000, 20000), 64)
    dout = torch.randn((20000, 136), device="cuda")
    t = Table(2000, 136, 20000)
    out = []
    for _ in range(3):
        grad = torch.empty((2000, 136), device="cuda")
        t.grad(ids, dout, FP32, grad, FP32)
        torch.cuda.synchronize()
        out.append(grad)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
    t.close()


def test_grad_against_differences():
    """The gradient of sum(w * lookup(table)) against differences of the library's own lookup.  Small whole numbers
    and a step of 1 make every value exact, so the two are equal."""
    torch, d = lib()
    rng = np.random.default_rng(7)
    rows, width, T = 7, 5, 60
    ids = ids_on(rng.integers(-1, rows + 1, T), 64)
    w = torch.from_numpy(rng.integers(-4, 5, (T, width)).astype(np.float32)).cuda()
    table = torch.from_numpy(rng.integers(-4, 5, (rows, width)).astype(np.float32)).cuda()
    grad = torch.empty_like(table)
    t = Table(rows, width, T)
    t.grad(ids, w, FP32, grad, FP32, 2.0)

    def loss(x):
        out = torch.empty((T, width), device="cuda")
        d.ddp_embedding_lookup(t.emb, T, ids.data_ptr(), 64, x.data_ptr(), FP32, width, 2.0, out.data_ptr(), FP32, width)
        return (out.double() * w.double()).sum().item()
    base = loss(table)
    for r in range(rows):
        for c in range(width):
            up = table.clone()
            up[r, c] += 1.0
            assert loss(up) - base == grad[r, c].item()
    t.close()


def test_grad_captured():
    """Replays of a captured call, with other tokens and eager work in between."""
    torch, _ = lib()
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(8)
    a, b = Table(300, 64, 3000, stream.cuda_stream), Table(300, 64, 3000)
    ids = ids_on(zipf(rng, 300, 3000), 64)
    dout = torch.randn((3000, 64), device="cuda", dtype=torch.bfloat16)
    one, two = torch.empty((300, 64), device="cuda"), torch.empty((300, 64), device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.grad(ids, dout, BF16, one, FP32)
    for k in range(4):
        ids.copy_(torch.from_numpy(zipf(rng, 300, 3000)))
        dout.normal_()
        one.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        b.grad(ids, dout, BF16, two, FP32)
        torch.cuda.synchronize()
        assert torch.equal(one, two), k
    a.close()
    b.close()


def test_a_workspace_that_does_not_fit():
    """2^22 tokens of a row of 2^20 columns ask for a terabyte.  The refusal is this call's alone: the next ones
    do not report it again."""
    torch, d = lib()
    with pytest.raises(d.DdpError) as e:
        d.ddp_embedding_create(0, 0, 1, 1 << 20, 1 << 22)
    assert e.value.code == d.DDP_ERR_HIP
    check_lookup(7, 40, [1, 2, 6], FP32, FP32)
    check_grad(7, 40, [1, 2, 6], FP32, FP32)


def test_destroy_waits_for_lookups():
    """A handle for lookups alone has no workspace to free; its outstanding work is waited for all the same."""
    torch, d = lib()
    rows, width, tokens = 64, 1024, 1 << 20
    stream = torch.cuda.Stream()
    table = torch.ones((rows, width), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(tokens, dtype=torch.int64, device="cuda")
    out = torch.zeros((tokens, width), dtype=torch.bfloat16, device="cuda")
    emb = d.ddp_embedding_create(0, stream.cuda_stream, rows, width, 0)
    torch.cuda.synchronize()
    for _ in range(50):                                       # some 20 ms
        d.ddp_embedding_lookup(emb, tokens, ids.data_ptr(), 64, table.data_ptr(), BF16, width, 3.0, out.data_ptr(), BF16, width)
    d.ddp_embedding_destroy(emb)
    assert stream.query(), "destroyed with work outstanding"
    assert (out == 3.0).all()


# Calls of more than 4096 tokens go by the sort whatever the table is; the rows' own tokens are at random places among ids
# that take no part.
LONG = 4500


def among_others(ids, seed, total=LONG):
    rng = np.random.default_rng(seed)
    out = np.where(np.arange(total) % 2 == 0, -1, 1 << 30)
    out[np.sort(rng.choice(total, len(ids), replace=False))] = ids
    return out


@pytest.mark.parametrize("lead", [0, 1, 31, 32, 33])
@pytest.mark.parametrize("tokens", [1, 31, 32, 33, 63, 64, 65, 96, 97, 4000])
def test_sorted_grad_of_one_row(tokens, lead):
    """Every length at which a row's tokens are split or end a part, starting everywhere in a window."""
    ids = np.concatenate([np.zeros(lead), np.full(tokens, 1), [3]])
    check_grad(5, 20, among_others(ids, tokens), FP32, FP32, poison=True)
    check_grad(5, 20, among_others(np.random.default_rng(lead).permutation(ids), tokens), BF16, FP32, add=True)


@pytest.mark.parametrize("lead", [0, 1, 127, 128])
def test_sorted_grad_of_long_windows(lead):
    """Few and wide rows: windows of 128 tokens."""
    lengths = (lead, 127, 129, 128, 256, 255, 257, 1, 0, 14000)
    ids = np.random.default_rng(lead).permutation(np.concatenate([np.full(n, r) for r, n in enumerate(lengths)]))
    check_grad(len(lengths), 2080, ids, FP32, BF16)


@pytest.mark.parametrize("lengths", [(33, 33, 33), (40, 1, 40), (32, 33, 31, 64), (1, 100, 1, 100), (33, 31, 33, 31, 1), (64, 64, 33, 0, 63)])
def test_sorted_grad_rows_that_meet_in_a_window(lengths):
    ids = np.concatenate([np.full(n, r) for r, n in enumerate(lengths)])
    for seed in range(2):
        mixed = among_others(np.random.default_rng(seed).permutation(ids), seed)
        check_grad(len(lengths), 24, mixed, BF16, BF16, seed=seed, poison=True)
        check_grad(len(lengths), 24, mixed, FP32, FP16, seed=seed, add=True)


@pytest.mark.parametrize("dout_dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("grad_dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("bits", [32, 64])
def test_sorted_grad_types(dout_dt, grad_dt, add, bits):
    rng = np.random.default_rng(2)
    check_grad(50, 130, zipf(rng, 50, LONG), dout_dt, grad_dt, add=add, bits=bits)
    check_grad(3000, 37, zipf(rng, 3000, LONG), dout_dt, grad_dt, add=add, bits=bits)
    check_grad(300, 3, zipf(rng, 300, LONG), dout_dt, grad_dt, add=add, bits=bits)


@pytest.mark.parametrize("padding", [-1, 0, 6])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("bits", [32, 64])
def test_sorted_grad_padding_is_not_read(padding, add, bits):
    rng = np.random.default_rng(3)
    ids = rng.integers(-3, 12, LONG + 1000)
    ids[7], ids[8] = (2 ** 31 - 1, -2 ** 31) if bits == 32 else (2 ** 40, -2 ** 50)
    check_grad(9, 77, ids, BF16, FP32, padding=padding, add=add, bits=bits, poison=True)
    ids = rng.integers(-100, 4000, LONG + 1000)
    check_grad(3900, 21, ids, FP16, FP16, padding=padding, add=add, bits=bits, poison=True)


@pytest.mark.parametrize("bits", [32, 64])
def test_sorted_grad_without_a_token_that_counts(bits):
    for rows in (9, 3000):
        got = check_grad(rows, 33, np.full(LONG, 4), FP32, FP16, padding=4, poison=True, bits=bits)
        assert (got == 0).all()
        check_grad(rows, 33, np.full(LONG, 4), FP32, FP16, padding=4, poison=True, add=True, bits=bits)
        check_grad(rows, 33, np.full(LONG, -1), FP32, FP16, add=True, bits=bits)
        got = check_grad(rows, 33, np.full(LONG, rows), BF16, BF16, poison=True, bits=bits)
        assert (got == 0).all()


@pytest.mark.parametrize("gaps,shifts", [((3, 0), (0, 1)), ((0, 5), (1, 3)), ((1, 1), (1, 0)), ((8, 8), (4, 4))])
@pytest.mark.parametrize("dt", [FP32, FP16, BF16])
def test_sorted_grad_strides_and_alignments(gaps, shifts, dt):
    rng = np.random.default_rng(4)
    for rows, width in ((61, 131), (2500, 259), (700, 5)):
        check_grad(rows, width, zipf(rng, rows, LONG), dt, dt, gaps=gaps, shifts=shifts)
        check_grad(rows, width, zipf(rng, rows, LONG), dt, FP32 if dt == BF16 else BF16, gaps=gaps, shifts=shifts, add=True)


def test_ids_at_any_element():
    """Ids that start in the middle of an 8- or 16-byte word, by either way through the tokens."""
    torch, d = lib()
    rng = np.random.default_rng(9)
    for bits in (32, 64):
        for tokens in (700, LONG):
            values = rng.integers(-2, 40, tokens)
            dout, grads = torch.randn((tokens, 24), device="cuda"), []
            t = Table(39, 24, tokens)
            for shift in (0, 1, 3):
                on, grad = ids_on(values, bits, shift), torch.empty((39, 24), device="cuda")
                torch.cuda.synchronize()
                t.grad(on, dout, FP32, grad, FP32, bits=bits)
                torch.cuda.synchronize()
                grads.append(grad)
            assert torch.equal(grads[0], grads[1]) and torch.equal(grads[0], grads[2])
            want, size = ops.embedding_grad(39, values, dout.double().cpu().numpy(), 1.5)
            assert (np.abs(grads[0].double().cpu().numpy() - want) <= (tokens + 3) * U * size).all()
            t.close()


@pytest.mark.parametrize("rows,width", [(300, 64), (5, 300), (20000, 21)])
def test_sorted_grad_captured(rows, width):
    """Replays of a captured call that sorts, with other tokens and eager work in between."""
    torch, _ = lib()
    tokens = 6000
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(8)
    a, b = Table(rows, width, tokens, stream.cuda_stream), Table(rows, width, tokens)
    ids = ids_on(zipf(rng, rows, tokens), 64)
    dout = torch.randn((tokens, width), device="cuda", dtype=torch.bfloat16)
    one, two = torch.empty((rows, width), device="cuda"), torch.empty((rows, width), device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.grad(ids, dout, BF16, one, FP32)
    for k in range(5):
        spread = zipf(rng, rows, tokens) if k % 2 else np.where(rng.random(tokens) < 0.5, rng.integers(-3, rows, tokens), k)
        ids.copy_(torch.from_numpy(spread))
        dout.normal_()
        one.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        b.grad(ids, dout, BF16, two, FP32)
        torch.cuda.synchronize()
        assert torch.equal(one, two), k
        want, size = ops.embedding_grad(rows, spread, dout.double().cpu().numpy(), 1.5)
        assert (np.abs(one.double().cpu().numpy() - want) <= (tokens + 3) * U * size).all(), k
    a.close()
    b.close()


@pytest.mark.parametrize("table_dt,out_dt", [(FP32, FP32), (FP32, BF16), (BF16, BF16), (FP16, FP32), (BF16, FP16)])
@pytest.mark.parametrize("width,tokens", [(1037, 2300), (67, 33000), (513, 4400)])
def test_lookup_of_more_than_the_caches_keep(table_dt, out_dt, width, tokens):
    """More than 4 MiB of rows are stored past the caches: odd widths, gaps and shifted bases."""
    rng = np.random.default_rng(width)
    assert width * tokens * (4 if out_dt == FP32 else 2) > 4 << 20
    check_lookup(41, width, rng.integers(-1, 42, tokens), table_dt, out_dt, 32, gaps=(1, 0), shifts=(1, 1))
    check_lookup(41, width, rng.integers(-1, 42, tokens), table_dt, out_dt, 64, gaps=(0, 3), shifts=(0, 3))


def check_whole(rows, width, ids, add=False, bits=64, max_tokens=None):
    """Small whole numbers: every sum is exact in binary32, whatever its order, so the gradient is compared with equality."""
    torch, d = lib()
    gen = torch.Generator(device="cuda").manual_seed(rows + width)
    ids = torch.as_tensor(ids, device="cuda")
    T = len(ids)
    dout = torch.randint(-3, 4, (T, width), generator=gen, device="cuda", dtype=torch.int8).bfloat16()
    grad = torch.full((rows + 1, width), 5.0, device="cuda")
    used = ((ids >= 0) & (ids < rows)).nonzero().reshape(-1)
    want = torch.full((rows, width), 5.0 if add else 0.0, device="cuda", dtype=torch.float64)
    if rows <= 8:
        for r in range(rows):
            for some in (ids == r).nonzero().reshape(-1).split(1 << 18):
                want[r] += 2.0 * dout[some].double().sum(0)
    else:
        for some in used.split(1 << 18):
            want.index_add_(0, ids[some].long(), 2.0 * dout[some].double())
    on = ids.to(torch.int64 if bits == 64 else torch.int32)
    emb = d.ddp_embedding_create(0, 0, rows, width, max_tokens or T)
    for _ in range(1 if add else 2):
        torch.cuda.synchronize()
        d.ddp_embedding_grad(emb, T, on.data_ptr(), bits, dout.data_ptr(), BF16, width, 2.0, -1, add, grad.data_ptr(), FP32, width)
    torch.cuda.synchronize()
    assert torch.equal(grad[:rows].double(), want) and (grad[rows] == 5.0).all()
    d.ddp_embedding_destroy(emb)


@pytest.mark.parametrize("rows,width", [((1 << 19) + 1, 12), ((1 << 20) + 3, 5), (1 << 23, 1), (40000, 1030), (30522, 64)])
@pytest.mark.parametrize("tokens", [1, 700, 4096, 4097, 20000])
@pytest.mark.parametrize("add", [False, True])
def test_grad_of_large_tables(rows, width, tokens, add):
    """Up to the largest table there can be, by either way through the tokens; blocks of the first have rows in pairs here."""
    rng = np.random.default_rng(rows)
    near = np.concatenate([[0, 1, rows - 1, rows - 2], rng.integers(0, 8, tokens)])[:tokens]
    check_whole(rows, width, rng.integers(-2, rows + 2, tokens), add)
    check_whole(rows, width, np.where(rng.random(tokens) < 0.5, near, rng.integers(0, rows, tokens)), add, bits=32)


@pytest.mark.parametrize("rows,width", [(1, 3), (2, 40), (5, 3), (700, 20), (30522, 9), (1 << 21, 2)])
@pytest.mark.parametrize("tokens", [524288, 524289, 1 << 22])
def test_grad_of_the_longest_calls(rows, width, tokens):
    """More chunks of tokens than a block of the sort has threads, up to the most tokens of a call."""
    rng = np.random.default_rng(tokens)
    check_whole(rows, width, zipf(rng, rows, tokens))
    check_whole(rows, width, rng.integers(-1, rows, tokens), bits=32)
    sparse = np.where(np.arange(tokens) % 4099 == 7, rng.integers(0, rows, tokens), -1)
    check_whole(rows, width, sparse)
    sparse[-100:] = rows - 1                     # of the last chunk alone
    check_whole(rows, width, sparse, add=True)


@pytest.mark.parametrize("tokens", [3, 1025])
@pytest.mark.parametrize("width", [1 << 20, (1 << 20) - 3])
def test_the_widest_rows(tokens, width):
    torch, d = lib()
    ids = np.arange(tokens) % 4 - 1
    check_whole(3, width, ids)
    check_whole(3, width, ids, add=True)
    table = torch.randint(-9, 9, (3, width), device="cuda").half()
    on, out = torch.as_tensor(ids[:7].copy(), device="cuda"), torch.full((len(ids[:7]), width), 7.0, device="cuda")
    emb = d.ddp_embedding_create(0, 0, 3, width, 0)
    torch.cuda.synchronize()
    d.ddp_embedding_lookup(emb, len(on), on.data_ptr(), 64, table.data_ptr(), FP16, width, 0.5, out.data_ptr(), FP32, width)
    torch.cuda.synchronize()
    want = torch.where((on >= 0)[:, None], table[on.clamp(min=0)].float() * 0.5, 0.0)
    assert torch.equal(out, want)
    d.ddp_embedding_destroy(emb)


def test_calls_of_no_tokens():
    """A lookup of none does nothing and needs no addresses; a gradient of none is zeros."""
    torch, d = lib()
    emb = d.ddp_embedding_create(0, 0, 5, 33, 10)
    d.ddp_embedding_lookup(emb, 0, 0, 64, 0, FP32, 33, 1.0, 0, BF16, 33)
    grad = torch.full((6, 33), 5.0, device="cuda")
    torch.cuda.synchronize()
    d.ddp_embedding_grad(emb, 0, 0, 32, 0, BF16, 33, 1.0, -1, True, grad.data_ptr(), FP32, 33)
    torch.cuda.synchronize()
    assert (grad == 5.0).all()
    d.ddp_embedding_grad(emb, 0, 0, 32, 0, BF16, 33, 1.0, -1, False, grad.data_ptr(), FP32, 33)
    torch.cuda.synchronize()
    assert (grad[:5] == 0.0).all() and (grad[5] == 5.0).all()
    d.ddp_embedding_destroy(emb)


def same_bits(got, want):
    """Equal, signs of zeros included; NaN is NaN, whatever its payload."""
    torch, _ = lib()
    whole = {torch.float32: torch.int32, torch.float16: torch.int16, torch.bfloat16: torch.int16}[got.dtype]
    nan = torch.isnan(want)
    return torch.equal(torch.isnan(got), nan) and torch.equal(got.view(whole)[~nan], want.view(whole)[~nan])


def every_pattern(dt):
    """[rows, 64]: all 16-bit patterns, or binary32 ones around every edge of the three types' ranges and roundings."""
    torch, _ = lib()
    if dt != FP32:
        return torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(torch_type(torch, dt)).view(-1, 64)
    edges = [0, 1, 2, 0x7FFF, 0x8000, 0x8001, 0xFFFF, 0x10000, 0x18000, 0x7FFFFF, 0x800000, 0x800001, 0x7F7FFFFF, 0x7F7F7FFF, 0x7F7F8000, 0x7F800000,
             0x7F800001, 0x7FC00000, 0x33000000, 0x33000001, 0x33800000, 0x387FC000, 0x387FE000, 0x38800000, 0x477FEFFF, 0x477FF000, 0x47800000,
             0x3F800000, 0x3F801000, 0x3F803000, 0x3F808000, 0x3F818000]
    rng = np.random.default_rng(12)
    bits = np.concatenate([np.array(edges), rng.integers(0, 0x7F800000, 8192 - 32)]).astype(np.uint32)
    return torch.from_numpy(np.concatenate([bits, bits | 0x80000000]).view(np.float32).copy()).view(-1, 64)


@pytest.mark.parametrize("table_dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("out_dt", [FP32, FP16, BF16])
@pytest.mark.parametrize("scale", [1.0, 3.0, 2.0 ** -20, -2.0 ** 30])
def test_lookup_and_grad_of_every_pattern(table_dt, out_dt, scale):
    """Subnormal numbers, the ends of the ranges, ties, infinities and NaN: one product in binary32, one rounding.  A gradient of one token
    a row is 0 + x, scaled (so that -0 becomes +0 times the scale)."""
    torch, d = lib()
    table = every_pattern(table_dt)
    rows, width = table.shape
    want = (table.float() * scale).to(torch_type(torch, out_dt))
    summed = ((table.float() + 0.0) * scale).to(torch_type(torch, out_dt))
    on = table.cuda()
    for tokens in (rows, 5000):
        ids = torch.cat([torch.randperm(rows, generator=torch.Generator().manual_seed(tokens)), torch.full((max(0, tokens - rows),), -1)])
        there, out = ids.cuda(), torch.empty((len(ids), width), dtype=torch_type(torch, out_dt), device="cuda")
        dout = torch.full((len(ids), width), float("nan"), dtype=table.dtype, device="cuda")
        dout[:rows] = on[there[:rows]]
        grad = torch.empty((rows, width), dtype=torch_type(torch, out_dt), device="cuda")
        emb = d.ddp_embedding_create(0, 0, rows, width, len(ids))
        torch.cuda.synchronize()
        d.ddp_embedding_lookup(emb, len(ids), there.data_ptr(), 64, on.data_ptr(), table_dt, width, scale, out.data_ptr(), out_dt, width)
        d.ddp_embedding_grad(emb, len(ids), there.data_ptr(), 64, dout.data_ptr(), table_dt, width, scale, -1, False, grad.data_ptr(), out_dt, width)
        torch.cuda.synchronize()
        assert same_bits(out[:rows].cpu(), want[ids[:rows]]) and (out[rows:] == 0).all()
        assert same_bits(grad.cpu(), summed)
        d.ddp_embedding_destroy(emb)
