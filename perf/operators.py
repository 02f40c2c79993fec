"""What a training program does around the gradient synchronization, operator by operator.

A case is one pass through one operator: the embedding lookup that opens a forward pass and its
gradient that closes the backward pass (the last tensor to become ready), and, on the averaged
gradients, the global norm and the AdamW step with states in 32 or in 8 bits.  With `own` the
calls are the library's, without it the same formulas in elementary torch operations, in 32 bits,
rounded once at the end.  The parameter lists are the repository's (the eight small tensors,
ResNet-50, BERT-large) or generated ones with the same make-up; the embedding sizes are those of
the BERT-large list's three tables, or generic.

Keys of a case:
  op        "lookup" | "embedding_grad" | "norm" | "adamw"
 embedding
  rows, width, tokens
  dtype     type of the table (lookup) or of the gradient that is written: 0 binary32, 1 binary16, 2 bfloat16
  flow      type of the rows that the lookup writes, or whose gradient comes in
  ids       bits of a token id, 32 or 64
  pad       share of the tokens that are padding: half of them the padding row 0, half of them -1
  spread    "zipf" (the row numbers are ranks of frequency) or "even"
  gap       further columns between two rows of what flows (a slice of a wider buffer)
  add       the gradient is added to what is there (a further micro-step)
 optimizer
  model     "tiny" | "resnet50" | "bert_large", or "generated" with tensors, elems (total), shape_seed
  param, grad   types of the parameters and gradients, copy = type of the forward pass's copy (-1: none)
  bits      bits of a state's element, 32 or 8
  clip      the gradients are clipped to a global norm (two calls: the norm, the step)
  dense     parameters and gradients packed without gaps, at element alignment
"""
import math
import random

import numpy as np
import torch

own = False

TORCH = {0: torch.float32, 1: torch.float16, 2: torch.bfloat16}
ESIZE = {0: 4, 1: 2, 2: 2}
BLOCK = 256                      # elements of a state that share a scale; tensors start at multiples of it
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
SIGMA = 1e-2                     # of a gradient's elements
STEPS = 10                       # steps taken before the pass
SCALE = 32.0                     # of the embedding: the square root of a width of 1024


def listed():
    return [
        # generating text: one token's row, read for the first layer
        {"name": "lookup_token", "op": "lookup", "rows": 30522, "width": 1024, "tokens": 1, "dtype": 2, "flow": 2,
         "ids": 64, "pad": 0.0, "spread": "zipf", "gap": 0},
        # a training batch of 32 sequences of 512 tokens; binary32 master table, bfloat16 activations
        {"name": "lookup_batch", "op": "lookup", "rows": 30522, "width": 1024, "tokens": 16384, "dtype": 0, "flow": 2,
         "ids": 64, "pad": 0.1, "spread": "zipf", "gap": 0},
        # the token-type table: two rows that share every gradient row of a short batch
        {"name": "grad_types", "op": "embedding_grad", "rows": 2, "width": 1024, "tokens": 512, "dtype": 0, "flow": 0,
         "ids": 64, "pad": 0.0, "spread": "even", "gap": 0, "add": False},
        # the word table, 8 sequences of 512 tokens: most rows of the gradient are zeros
        {"name": "grad_words", "op": "embedding_grad", "rows": 30522, "width": 1024, "tokens": 4096, "dtype": 0,
         "flow": 2, "ids": 64, "pad": 0.1, "spread": "zipf", "gap": 0, "add": False},
        # a long batch, the gradient in bfloat16
        {"name": "grad_long", "op": "embedding_grad", "rows": 30522, "width": 1024, "tokens": 65536, "dtype": 2,
         "flow": 2, "ids": 32, "pad": 0.1, "spread": "zipf", "gap": 0, "add": False},
        # odd sizes, rows of a wider buffer, added to the gradient of the micro-steps before
        {"name": "grad_ragged", "op": "embedding_grad", "rows": 32003, "width": 771, "tokens": 20011, "dtype": 0,
         "flow": 1, "ids": 64, "pad": 0.05, "spread": "zipf", "gap": 5, "add": True},
        # the global norm by itself, for a program that has its own step
        {"name": "norm_resnet50", "op": "norm", "model": "resnet50", "grad": 0, "dense": False},
        {"name": "norm_bert_large_bf16", "op": "norm", "model": "bert_large", "grad": 2, "dense": False},
        # the smallest model: the calls' own cost
        {"name": "adamw_tiny", "op": "adamw", "model": "tiny", "param": 0, "grad": 0, "copy": -1, "bits": 32,
         "clip": True, "dense": False},
        # mixed precision: bfloat16 gradients, binary32 master parameters, bfloat16 copy for the next forward pass
        {"name": "adamw_bert_large", "op": "adamw", "model": "bert_large", "param": 0, "grad": 2, "copy": 2, "bits": 32,
         "clip": True, "dense": False},
        # 8-bit states: an odd list packed without gaps, and the large model; the pass ends with the states read
        # out as the values they stand for, as for a checkpoint
        {"name": "adamw8_ragged", "op": "adamw", "model": "generated", "tensors": 90, "elems": 3000001, "shape_seed": 5,
         "param": 0, "grad": 1, "copy": -1, "bits": 8, "clip": False, "dense": True},
        {"name": "adamw8_bert_large", "op": "adamw", "model": "bert_large", "param": 0, "grad": 2, "copy": 2, "bits": 8,
         "clip": False, "dense": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["lookup", "embedding_grad", "embedding_grad", "norm", "adamw", "adamw", "adamw"])
    if op in ("lookup", "embedding_grad"):
        case = {"op": op, "width": _log_uniform(rng, 16, 4096), "dtype": rng.choice([0, 0, 1, 2]),
                "flow": rng.choice([0, 1, 2, 2]), "ids": rng.choice([32, 64]),
                "pad": rng.choice([0.0, 0.0, 0.1, 0.3]), "spread": rng.choice(["zipf", "zipf", "even"]),
                "gap": rng.choice([0, 0, 0, 8, 5])}
        if rng.random() < 0.5:
            case["width"] = max(16, case["width"] // 64 * 64)
        case["rows"] = _log_uniform(rng, 2, min(131072, 400000000 // case["width"]))
        case["tokens"] = _log_uniform(rng, 1, min(131072, 200000000 // case["width"]))
        if op == "embedding_grad":
            case["add"] = rng.random() < 0.25
        return case
    case = {"op": op, "model": "generated", "elems": _log_uniform(rng, 5000, 300000000), "tensors": rng.randrange(2, 400),
            "shape_seed": rng.randrange(1 << 20), "grad": rng.choice([0, 0, 1, 2, 2]), "dense": rng.random() < 0.3}
    if op == "adamw":
        case["bits"] = rng.choice([32, 32, 8])
        case["param"] = rng.choice([0, 0, 0, case["grad"]])
        case["copy"] = rng.choice([-1, 1, 2, 2]) if case["param"] == 0 else -1
        # (the steps of the norm's sum would show in the 8-bit codes: there the program scales by a number it has)
        case["clip"] = case["bits"] == 32 and rng.random() < 0.7
    return case


# ---- sizes ----

def _numel(case):
    if case["model"] != "generated":
        import workloads
        return workloads.numel_of(workloads.WORKLOAD_SHAPES[case["model"]]())
    # weights whose sizes spread over three decades, each followed by a small vector
    rng = random.Random(case["shape_seed"])
    size = [10.0 ** rng.uniform(0.0, 3.0) if i % 2 == 0 else 0.02 * 10.0 ** rng.uniform(0.0, 1.5)
            for i in range(case["tensors"])]
    scale = case["elems"] / sum(size)
    return [max(1, int(s * scale)) for s in size]


def _starts(numel):
    """Where each tensor starts in a state, and the state's elements."""
    at, total = [], 0
    for n in numel:
        at.append(total)
        total += (n + BLOCK - 1) // BLOCK * BLOCK
    return at, total


def _up(x, to):
    return (x + to - 1) // to * to


def _unique(case):
    """Rows that the tokens are expected to name, and the share of the tokens that are no padding row."""
    V, T = case["rows"], case["tokens"] * (1.0 - case["pad"])
    k = np.arange(V, dtype=np.float64)
    p = np.log1p(1.0 / (k + 1.0)) / math.log(V + 1.0) if case["spread"] == "zipf" else np.full(V, 1.0 / V)
    return float((1.0 - np.exp(-T * p)).sum())


def work(case):
    if case["op"] in ("lookup", "embedding_grad"):
        T, D, V, idb = case["tokens"], case["width"], case["rows"], case["ids"] // 8
        kept, rows = T * (1.0 - case["pad"]), min(_unique(case), float(V))
        es, fs = ESIZE[case["dtype"]], ESIZE[case["flow"]]
        if case["op"] == "lookup":
            return {"bytes": T * idb + D * (rows * es + T * fs), "flops": T * D}
        out = rows * 2 * es if case["add"] else V * es
        return {"bytes": T * idb + D * (kept * fs + out), "flops": kept * D + rows * D}
    numel = _numel(case)
    n, gs = sum(numel), ESIZE[case["grad"]]
    if case["op"] == "norm":
        return {"bytes": n * gs + 4, "flops": 2 * n}
    cs = ESIZE[case["copy"]] if case["copy"] >= 0 else 0
    each = gs + 2 * ESIZE[case["param"]] + cs
    if case["bits"] == 32:
        each += 16
    else:
        each += 2 * 2 * (1 + 4 / BLOCK) + 2 * 4        # codes and scales, both ways; the values read out
    return {"bytes": n * each, "flops": n * (14 if case["bits"] == 32 else 34) + (2 * n if case["clip"] else 0)}


# ---- inputs ----

class _State:
    def __init__(self):
        self.handle = self.free = None

    def __del__(self):
        if self.handle is not None:
            self.free(self.handle)
            self.handle = None


def _gen(seed, salt):
    g = torch.Generator("cuda")
    g.manual_seed((seed * 1000003 + salt * 4099) % (1 << 62))
    return g


def _normal(shape, dtype, seed, salt, sigma):
    x = torch.empty(shape, dtype=dtype, device="cuda")
    x.normal_(0.0, sigma, generator=_gen(seed, salt))
    return x


def _tokens(case, seed):
    V, T = case["rows"], case["tokens"]
    u = torch.rand(T, generator=_gen(seed, 1), device="cuda", dtype=torch.float64)
    ids = torch.exp(u * math.log(V + 1.0)) - 1.0 if case["spread"] == "zipf" else u * V
    ids = ids.long().clamp_(0, V - 1)
    if case["pad"]:
        w = torch.rand(T, generator=_gen(seed, 2), device="cuda")
        ids = torch.where(w < case["pad"] / 2, torch.zeros_like(ids), ids)
        ids = torch.where(w > 1.0 - case["pad"] / 2, torch.full_like(ids, -1), ids)
    return ids if case["ids"] == 64 else ids.int()


def _prepare_embedding(case, seed):
    st = _State()
    st.case = case
    V, D, T, gap = case["rows"], case["width"], case["tokens"], case["gap"]
    st.ids = _tokens(case, seed)
    st.padding = 0 if case["pad"] else -1
    if case["op"] == "lookup":
        st.table = _normal((V, D), TORCH[case["dtype"]], seed, 3, 0.02)
        st.out = torch.zeros((T, D + gap), dtype=TORCH[case["flow"]], device="cuda")[:, :D]
    else:
        st.dout = _normal((T, D + gap), TORCH[case["flow"]], seed, 4, SIGMA)[:, :D]
        st.grad = _normal((V, D), TORCH[case["dtype"]], seed, 5, SIGMA)
    if own:
        import paper_2006_15704_amd as ddp
        st.handle = ddp.ddp_embedding_create(0, torch.cuda.current_stream().cuda_stream, V, D,
                                             T if case["op"] == "embedding_grad" else 0)
        st.free = ddp.ddp_embedding_destroy
    return st


def _buffers(case, numel, seed):
    """Flat buffers: (where each tensor starts in parameters and gradients, gradients, parameters or None)."""
    at, total = _starts(numel)
    if case["dense"]:
        at, total = [], 0
        for n in numel:
            at.append(total)
            total += n
    g = _normal(total, TORCH[case["grad"]], seed, 11, SIGMA)
    p = _normal(total, TORCH[case["param"]], seed, 12, 0.05) if case["op"] == "adamw" else None
    if not case["dense"]:
        real = _real(numel)
        g.mul_(real)
        if p is not None:
            p.mul_(real)
    return at, g, p


def _per_tensor(values, numel, dtype):
    """One value a tensor, at every element of the tensors' places in a state (0 between them)."""
    at, total = _starts(numel)
    room = np.diff(np.append(at, total))
    each = np.repeat(np.stack([np.asarray(values, dtype=np.float64), np.zeros(len(numel))], 1).reshape(-1),
                     np.stack([numel, room - np.asarray(numel)], 1).reshape(-1)) if total <= 1 << 16 else None
    if each is not None:
        return torch.from_numpy(each).to("cuda", dtype)
    count = torch.tensor(np.stack([numel, room - np.asarray(numel)], 1).reshape(-1), device="cuda")
    value = torch.tensor(np.stack([np.asarray(values, dtype=np.float64), np.zeros(len(numel))], 1).reshape(-1), device="cuda")
    return torch.repeat_interleave(value.to(dtype), count, output_size=total)


def _real(numel):
    return _per_tensor([1.0] * len(numel), numel, torch.bool)


def _decays(numel):
    """Vectors and biases do not decay: the shorter tensors of each list."""
    return [0.0 if n <= 4096 else 1.0 for n in numel]


def _prepare_optimizer(case, seed):
    st = _State()
    st.case, st.numel = case, _numel(case)
    at, st.g, st.p = _buffers(case, st.numel, seed)
    starts, total = _starts(st.numel)
    st.norm = torch.zeros(1, dtype=torch.float32, device="cuda")
    st.where = _real(st.numel).nonzero().reshape(-1) if case["dense"] else None   # of packed elements in a state
    st.max_norm = 0.5 * SIGMA * math.sqrt(sum(st.numel))        # clips: the norm is about twice that
    if case["op"] == "adamw":
        es = case["bits"] // 8
        # a state: 256 bytes with the number of steps, then first moments, second moments, and with 8 bits their scales
        st.state = torch.zeros(_state_bytes(case, total), dtype=torch.uint8, device="cuda")
        st.step = st.state[:8].view(torch.int64)
        st.step.fill_(STEPS)
        real = _real(st.numel)
        st.decay = _per_tensor(_decays(st.numel), st.numel, torch.float32)
        a = 256
        if case["bits"] == 32:
            st.m = st.state[a:a + 4 * total].view(torch.float32)
            st.v = st.state[a + 4 * total:a + 8 * total].view(torch.float32)
            st.m.normal_(0.0, SIGMA / 3, generator=_gen(seed, 13)).mul_(real)
            st.v.normal_(0.0, SIGMA, generator=_gen(seed, 14)).square_().add_(1e-2 * SIGMA * SIGMA).mul_(real)
        else:
            blocks = total // BLOCK
            st.m8 = st.state[a:a + total].view(torch.int8)
            st.v8 = st.state[a + total:a + 2 * total]
            b = a + 2 * total
            st.m_top = st.state[b:b + 4 * blocks].view(torch.float32)
            b += _up(4 * blocks, 256)
            st.v_top = st.state[b:b + 4 * blocks].view(torch.float32)
            st.m8.copy_(torch.randint(-127, 128, (total,), generator=_gen(seed, 13), device="cuda", dtype=torch.int8)).mul_(real)
            st.v8.copy_(torch.randint(64, 256, (total,), generator=_gen(seed, 14), device="cuda", dtype=torch.uint8)).mul_(real)
            st.m_top.uniform_(0.2 * SIGMA, SIGMA, generator=_gen(seed, 15))
            st.v_top.uniform_(SIGMA ** 2, 9 * SIGMA ** 2, generator=_gen(seed, 16))
            st.m = torch.zeros(total, dtype=torch.float32, device="cuda")      # the states as values
            st.v = torch.zeros(total, dtype=torch.float32, device="cuda")
        st.copy = torch.zeros_like(st.p, dtype=TORCH[case["copy"]]) if case["copy"] >= 0 else None
    if own:
        import paper_2006_15704_amd as ddp
        st.handle = ddp.ddp_opt_create(0, torch.cuda.current_stream().cuda_stream)
        st.free = ddp.ddp_opt_destroy
        n = len(st.numel)

        def ptrs(x):
            return None if x is None else [x.data_ptr() + o * x.element_size() for o in at]

        ddp.ddp_opt_register(st.handle, st.numel, [case.get("param", 0)] * n, ptrs(st.p), [case["grad"]] * n, ptrs(st.g))
        if case["op"] == "adamw":
            ddp.ddp_opt_set_groups(st.handle, None, _decays(st.numel))
            if st.copy is not None:
                ddp.ddp_opt_set_copies(st.handle, [case["copy"]] * n, ptrs(st.copy))
            ddp.ddp_opt_set_state(st.handle, ddp.DDP_STATE_FP32 if case["bits"] == 32 else ddp.DDP_STATE_8BIT,
                                  st.state.data_ptr(), st.state.numel())
    return st


def _state_bytes(case, total):
    if case["bits"] == 32:
        return 256 + 8 * total
    return 256 + 2 * total + 2 * _up(4 * (total // BLOCK), 256)


def prepare(case, seed):
    if case["op"] in ("lookup", "embedding_grad"):
        return _prepare_embedding(case, seed)
    return _prepare_optimizer(case, seed)


# ---- passes ----

def run(st):
    op = st.case["op"]
    if own:
        import paper_2006_15704_amd as ddp
        if op == "lookup":
            return _own_lookup(ddp, st)
        if op == "embedding_grad":
            return _own_embedding_grad(ddp, st)
        return _own_norm(ddp, st) if op == "norm" else _own_adamw(ddp, st)
    if op == "lookup":
        return _plain_lookup(st)
    if op == "embedding_grad":
        return _plain_embedding_grad(st)
    return _plain_norm(st) if op == "norm" else _plain_adamw(st)


def _own_lookup(ddp, st):
    c = st.case
    ddp.ddp_embedding_lookup(st.handle, c["tokens"], st.ids.data_ptr(), c["ids"], st.table.data_ptr(), c["dtype"],
                             st.table.stride(0), SCALE, st.out.data_ptr(), c["flow"], st.out.stride(0))
    return st.out


def _own_embedding_grad(ddp, st):
    c = st.case
    ddp.ddp_embedding_grad(st.handle, c["tokens"], st.ids.data_ptr(), c["ids"], st.dout.data_ptr(), c["flow"],
                           st.dout.stride(0), SCALE, st.padding, c["add"], st.grad.data_ptr(), c["dtype"],
                           st.grad.stride(0))
    return st.grad


def _own_norm(ddp, st):
    ddp.ddp_opt_grad_norm(st.handle, 1.0, st.norm.data_ptr())
    return st.norm


def _own_adamw(ddp, st):
    if st.case["clip"]:
        ddp.ddp_opt_grad_norm(st.handle, 1.0, st.norm.data_ptr())
    ddp.ddp_opt_adamw_step(st.handle, LR, BETA1, BETA2, EPS, DECAY, 1.0, st.max_norm if st.case["clip"] else 0.0)
    if st.case["bits"] == 8:
        ddp.ddp_opt_read_state(st.handle, st.m.data_ptr(), st.v.data_ptr())
    return _optimizer_outputs(st)


def _optimizer_outputs(st):
    out = {"param": st.p, "m": st.m, "v": st.v}
    if st.copy is not None:
        out["copy"] = st.copy
    if st.case["clip"]:
        out["norm"] = st.norm
    return out


def _plain_lookup(st):
    named = (st.ids >= 0) & (st.ids < st.case["rows"])
    rows = st.table[torch.where(named, st.ids, 0).long()].float() * SCALE
    st.out.copy_(torch.where(named[:, None], rows, 0.0))
    return st.out


def _plain_embedding_grad(st):
    c = st.case
    kept = (st.ids >= 0) & (st.ids < c["rows"]) & (st.ids != st.padding)
    src = torch.where(kept[:, None], st.dout.float(), 0.0)
    total = torch.zeros((c["rows"], c["width"]), dtype=torch.float32, device="cuda")
    total.index_add_(0, torch.where(kept, st.ids, 0).long(), src)
    total *= SCALE
    if c["add"]:
        total += st.grad
    st.grad.copy_(total)
    return st.grad


def _plain_norm(st):
    g = st.g.float()
    st.norm.copy_((g * g).sum().sqrt())
    return st.norm


def _spread(st, x):
    """Packed elements at their places in a state."""
    if st.where is None:
        return x.float()
    wide = torch.zeros(st.decay.numel(), dtype=torch.float32, device="cuda")
    wide[st.where] = x.float()
    return wide


def _plain_adamw(st):
    c = st.case
    g, p = _spread(st, st.g), _spread(st, st.p)
    if c["clip"]:
        st.norm.copy_((g * g).sum().sqrt())
        g = g * (st.max_norm / (st.norm + 1e-6)).clamp(max=1.0)
    if c["bits"] == 32:
        m, v = st.m, st.v
    else:
        code = st.m8.float().view(-1, BLOCK)
        m = (st.m_top[:, None] * (code * code.abs() * (1.0 / 127 ** 2))).view(-1)
        code = st.v8.float().view(-1, BLOCK)
        v = (st.v_top[:, None] * ((code * code) * (code * code) * (1.0 / 255 ** 4))).view(-1)
    st.step += 1
    t = st.step.double()
    left1, left2 = (1.0 - BETA1 ** t).float(), (1.0 - BETA2 ** t).float()
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    p = p * (1.0 - LR * DECAY * st.decay) - (LR / left1) * (m / (v.sqrt() / left2.sqrt() + EPS))
    if st.where is not None:
        p = p[st.where]
    st.p.copy_(p)
    if st.copy is not None:
        st.copy.copy_(p)
    if c["bits"] == 32:
        st.m.copy_(m)
        st.v.copy_(v)
        return _optimizer_outputs(st)
    # first moments: the block's largest absolute value times (k / 127)^2 with the sign of k; second moments: the
    # block's largest times (k / 255)^4, and never 0 for what is not; the nearest k in the root's scale
    m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
    m_top, v_top = m.abs().amax(1, True), v.amax(1, True)
    q = (m.abs() * torch.where(m_top > 0, 1.0 / m_top, 0.0)) * float(127 ** 2)
    k = (q.sqrt() + 0.5).floor()
    k = k + ((k + 0.5) * (k + 0.5) <= q).float() - (((k - 0.5) * (k - 0.5) > q) & (k > 0)).float()
    k = k.clamp(max=127.0) * torch.where(m < 0, -1.0, 1.0)
    st.m8.copy_(k.view(-1))
    st.m_top.copy_(m_top.view(-1))
    st.m.copy_((m_top * (k * k.abs() * (1.0 / 127 ** 2))).view(-1))
    q = (v * torch.where(v_top > 0, 1.0 / v_top, 0.0)) * float(255 ** 4)
    k = (q.sqrt().sqrt() + 0.5).floor()
    up, down = (k + 0.5) * (k + 0.5), (k - 0.5) * (k - 0.5)
    k = k + (up * up <= q).float() - ((down * down > q) & (k > 0)).float()
    k = torch.maximum(k.clamp(max=255.0), (v > 0).float())
    st.v8.copy_(k.view(-1))
    st.v_top.copy_(v_top.view(-1))
    st.v.copy_((v_top * ((k * k) * (k * k) * (1.0 / 255 ** 4))).view(-1))
    return _optimizer_outputs(st)


# ---- the same in 64 bits, from the definitions ----

def exact(case, seed):
    if case["op"] == "lookup":
        ids = _tokens(case, seed).long()
        rows = _normal((case["rows"], case["width"]), TORCH[case["dtype"]], seed, 3, 0.02).double() * SCALE
        rows = torch.cat([rows, torch.zeros((1, case["width"]), dtype=torch.float64, device="cuda")])
        return rows[torch.where(ids < 0, case["rows"], ids)]
    if case["op"] == "embedding_grad":
        T, D = case["tokens"], case["width"]
        ids = _tokens(case, seed).long()
        use = (ids >= (1 if case["pad"] else 0)).nonzero().reshape(-1)
        dout = _normal((T, D + case["gap"]), TORCH[case["flow"]], seed, 4, SIGMA)[:, :D]
        total = torch.zeros((case["rows"], D), dtype=torch.float64, device="cuda")
        for some in use.split(16384):
            total.index_add_(0, ids[some], dout[some].double() * SCALE)
        if case["add"]:
            total += _normal((case["rows"], D), TORCH[case["dtype"]], seed, 5, SIGMA).double()
        return total
    numel = _numel(case)
    at, flat_g, flat_p = _buffers(case, numel, seed)
    if case["op"] == "norm":
        return sum((x.double() ** 2).sum() for x in flat_g.split(1 << 24)).sqrt().reshape(1)
    st = _prepare_optimizer_inputs(case, seed)
    clip = 1.0
    out = {"param": torch.zeros(flat_p.shape, dtype=torch.float64, device="cuda")}
    if case["clip"]:
        norm = sum((x.double() ** 2).sum() for x in flat_g.split(1 << 24)).sqrt()
        clip = torch.clamp(st.max_norm / (norm + 1e-6), max=1.0)
        out["norm"] = norm.reshape(1)
    starts, total = _starts(numel)
    out["m"] = torch.zeros(total, dtype=torch.float64, device="cuda")
    out["v"] = torch.zeros(total, dtype=torch.float64, device="cuda")
    t = STEPS + 1
    for i, n in enumerate(numel):
        s, a = slice(starts[i], starts[i] + n), slice(at[i], at[i] + n)
        g = flat_g[a].double() * clip
        if case["bits"] == 32:
            m, v = st.m[s].double(), st.v[s].double()
        else:
            b = slice(starts[i] // BLOCK, (starts[i] + n + BLOCK - 1) // BLOCK)
            m = _held(st.m8[s].double() / 127, st.m_top[b], 2)
            v = _held(st.v8[s].double() / 255, st.v_top[b], 4)
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g * g
        rate = m / (1 - BETA1 ** t) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
        p = flat_p[a].double()
        out["param"][a] = p - LR * DECAY * _decays([n])[0] * p - LR * rate
        if case["bits"] == 8:
            m, v = _rounded(m, 127, 2, 0), _rounded(v, 255, 4, 1)
        out["m"][s], out["v"][s] = m, v
    if case["copy"] >= 0:
        out["copy"] = out["param"]
    return out


def _prepare_optimizer_inputs(case, seed):
    global own
    was, own = own, False
    try:
        return _prepare_optimizer(case, seed)
    finally:
        own = was


def _held(part, top, power):
    return torch.sign(part) * part.abs() ** power * top.double().repeat_interleave(BLOCK)[:part.numel()]


def _rounded(x, levels, power, least):
    rows = torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)
    top = rows.abs().amax(1, keepdim=True)
    share = torch.where(top > 0, rows.abs() / top, torch.zeros_like(rows))
    k = torch.floor(share ** (1.0 / power) * levels + 0.5)
    k = torch.where(share > 0, k.clamp(min=least), k)
    return (torch.sign(rows) * (k / levels) ** power * top).view(-1)[:x.numel()]
