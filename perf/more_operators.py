"""What surrounds the matrix products of a transformer layer in training, operator by operator.

A case is one pass through one operator whose small parameters all tokens share: the layer norm with its residual sum,
forward and backward; the learned relative position bias by buckets and its gradient; the routing of tokens to experts, its
gradient, and the step of the balance bias by the replicas' counts.  With `own` the calls are the library's, without it
the same formulas in elementary torch operations, in 32 bits (64 for what is compared, and for the long sums), rounded
once at the end.

Keys of a case:
  op        "norm" | "norm_grad" | "bias" | "bias_grad" | "route" | "route_grad"
  dtype     type of what comes in (x, scores, logits): 0 binary32, 1 binary16, 2 bfloat16
  gap       further columns between two rows of it (a slice of a wider buffer)
 norm, norm_grad
  rows, width
  flow      type of y (its gradient)
  param     type of gamma and beta
  residual  x + residual is normalized, and written (forward); what flows back along the sum is added to dx (backward)
  stats     the forward pass writes mean and 1 / deviation (training)
  grad, add type of the parameters' gradients; they are added to what is there (a further micro-step)
 bias, bias_grad
  batch, heads, queries, keys, offset   (offset: position of the first query, counted from the first key)
  buckets, exact, distance, both        (both: buckets of their own for keys behind the query)
  param     type of the table (bias) or of its gradient (bias_grad)
  causal    keys behind the query are masked
  ragged    sequences end at lengths of their own
  add       to the scores that are there (bias), to the gradient that is there (bias_grad)
 route, route_grad
  tokens, experts, chosen, groups, kept, top    (top: largest keys of a group that are its score)
  score     0 softmax, 1 sigmoid;  renorm: the chosen weights sum up to `scale`;  scale
  param     type of the weights (of their gradient)
  replicas  0, or the balance bias is moved by the counts of so many replicas
"""
import math

import torch

own = False

TORCH = {0: torch.float32, 1: torch.float16, 2: torch.bfloat16}
ESIZE = {0: 4, 1: 2, 2: 2}
EPS = 1e-5
RATE = 1e-3                      # of the balance bias
LOWEST = -1e9                    # what a masked score is set to; bfloat16 and binary32 hold it


def listed():
    return [
        # generating text: one token
        {"name": "norm_token", "op": "norm", "rows": 1, "width": 1024, "dtype": 2, "flow": 2, "param": 0, "residual": False,
         "stats": False, "gap": 0},
        # a training batch of 32 sequences of 512 tokens, with the residual sum
        {"name": "norm_batch", "op": "norm", "rows": 16384, "width": 1024, "dtype": 2, "flow": 2, "param": 0, "residual": True,
         "stats": True, "gap": 0},
        # odd sizes, binary32 stream and 16-bit activations, a further micro-step
        {"name": "norm_grad_ragged", "op": "norm_grad", "rows": 20011, "width": 771, "dtype": 0, "flow": 1, "param": 0,
         "residual": False, "gap": 5, "grad": 0, "add": True},
        # a long batch of a wide layer
        {"name": "norm_grad_wide", "op": "norm_grad", "rows": 32768, "width": 4096, "dtype": 2, "flow": 2, "param": 2,
         "residual": True, "gap": 0, "grad": 0, "add": False},
        # one new token against what came before it
        {"name": "bias_token", "op": "bias", "batch": 1, "heads": 16, "queries": 1, "keys": 4097, "offset": 4096, "buckets": 32,
         "exact": 16, "distance": 128, "both": False, "dtype": 2, "param": 0, "causal": True, "ragged": False, "add": False,
         "gap": 0},
        # the bias of a long causal layer, for any attention that takes one
        {"name": "bias_causal", "op": "bias", "batch": 1, "heads": 16, "queries": 4096, "keys": 4096, "offset": 0,
         "buckets": 32, "exact": 16, "distance": 128, "both": False, "dtype": 2, "param": 0, "causal": True,
         "ragged": False, "add": False, "gap": 0},
        # an encoder's scores, sequences of 512 tokens at most
        {"name": "bias_grad_batch", "op": "bias_grad", "batch": 8, "heads": 16, "queries": 512, "keys": 512, "offset": 0,
         "buckets": 32, "exact": 8, "distance": 128, "both": True, "dtype": 0, "param": 0, "causal": False, "ragged": True,
         "add": True, "gap": 0},
        {"name": "bias_grad_long", "op": "bias_grad", "batch": 2, "heads": 16, "queries": 4096, "keys": 4096, "offset": 0,
         "buckets": 32, "exact": 16, "distance": 128, "both": False, "dtype": 2, "param": 0, "causal": True,
         "ragged": False, "add": False, "gap": 0},
        # one token; a training batch with groups, balance bias and the counts of eight replicas
        {"name": "route_token", "op": "route", "tokens": 1, "experts": 64, "chosen": 2, "groups": 1, "kept": 1, "top": 1,
         "score": 0, "renorm": True, "scale": 1.0, "dtype": 2, "param": 0, "replicas": 0, "gap": 0},
        {"name": "route_batch", "op": "route", "tokens": 65536, "experts": 256, "chosen": 8, "groups": 8, "kept": 4, "top": 2,
         "score": 1, "renorm": True, "scale": 2.5, "dtype": 0, "param": 0, "replicas": 8, "gap": 0},
        # odd sizes, every expert in one group
        {"name": "route_grad_ragged", "op": "route_grad", "tokens": 20011, "experts": 60, "chosen": 4, "groups": 1, "kept": 1,
         "top": 1, "score": 0, "renorm": False, "scale": 1.0, "dtype": 0, "param": 2, "gap": 3},
        {"name": "route_grad_batch", "op": "route_grad", "tokens": 65536, "experts": 256, "chosen": 8, "groups": 8, "kept": 4,
         "top": 2, "score": 1, "renorm": True, "scale": 2.5, "dtype": 2, "param": 0, "gap": 0},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "bias", "bias_grad", "bias_grad", "route", "route_grad"])
    case = {"op": op, "dtype": rng.choice([0, 0, 1, 2, 2]), "gap": rng.choice([0, 0, 0, 8, 3])}
    if op in ("norm", "norm_grad"):
        case["width"] = _log_uniform(rng, 16, 16384)
        if rng.random() < 0.6:
            case["width"] = max(16, case["width"] // 64 * 64)
        case["rows"] = _log_uniform(rng, 1, 60000000 // case["width"])
        case["flow"] = case["dtype"] if case["dtype"] else rng.choice([0, 1, 2])
        case["param"] = rng.choice([0, 0, case["dtype"]])
        case["residual"] = rng.random() < 0.5
        if op == "norm":
            case["stats"] = rng.random() < 0.7
        else:
            case["grad"], case["add"] = rng.choice([0, 0, case["dtype"]]), rng.random() < 0.25
        return case
    if op in ("bias", "bias_grad"):
        case["both"] = rng.random() < 0.5
        sides = 2 if case["both"] else 1
        case["buckets"] = sides * _log_uniform(rng, 2, 128)
        n = case["buckets"] // sides
        case["exact"] = rng.choice([max(1, n // 2), max(1, n // 2), n, rng.randrange(1, n + 1)])
        case["distance"] = case["exact"] + _log_uniform(rng, 8, 2000)
        case["heads"] = _log_uniform(rng, 1, 64)
        case["queries"], case["keys"] = _log_uniform(rng, 1, 8192), _log_uniform(rng, 1, 8192)
        if rng.random() < 0.6:
            case["keys"] = max(case["queries"], case["keys"])
        most = (1 << (29 if op == "bias" else 30)) // (ESIZE[case["dtype"]] * case["heads"] * case["queries"] * (case["keys"] + case["gap"]))
        if most < 1:
            case["queries"], most = max(1, case["queries"] // 32), 1
        case["batch"] = _log_uniform(rng, 1, min(32, most))
        case["offset"] = rng.choice([0, case["keys"] - case["queries"], case["keys"] // 2])
        case["param"] = rng.choice([0, 0, case["dtype"]])
        case["causal"], case["ragged"], case["add"] = rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.4
        return case
    case["experts"] = _log_uniform(rng, 4, 512)
    if rng.random() < 0.6:
        case["experts"] = max(4, case["experts"] // 8 * 8)
    case["groups"] = rng.choice([g for g in (1, 1, 1, 2, 4, 8) if case["experts"] % g == 0 and case["experts"] // g >= 2])
    case["kept"] = rng.randrange(1, case["groups"] + 1)
    case["top"] = rng.choice([1, 2])
    case["chosen"] = _log_uniform(rng, 1, min(16, case["kept"] * (case["experts"] // case["groups"])))
    case["tokens"] = _log_uniform(rng, 1, min(131072, 16777216 // case["experts"]))
    case["score"], case["renorm"], case["scale"] = rng.choice([0, 1]), rng.random() < 0.6, rng.choice([1.0, 2.5])
    case["param"] = rng.choice([0, 0, 2])
    if op == "route":
        case["replicas"] = rng.choice([0, 0, 4])
    return case


def _seen(case):
    """Places of the scores that are visible (with ragged lengths, about: they are drawn between a half and all)."""
    Q, K, o = case["queries"], case["keys"], case["offset"]
    seen = float(Q * K)
    if case["causal"]:
        seen = float(sum(min(max(i + o + 1, 0), K) for i in range(Q)))
    if case["ragged"]:
        seen *= 0.75 if case["op"] == "bias" else 0.5625
    return seen * case["batch"] * case["heads"]


def work(case):
    op, es = case["op"], ESIZE[case["dtype"]]
    if op in ("norm", "norm_grad"):
        T, D, fs, ps = case["rows"], case["width"], ESIZE[case["flow"]], ESIZE[case["param"]]
        if op == "norm":
            return {"bytes": T * D * (es + fs + (2 * es if case["residual"] else 0)) + (8 * T if case["stats"] else 0) + 2 * D * ps,
                    "flops": T * D * (9 if case["residual"] else 8)}
        gs = ESIZE[case["grad"]] * (2 if case["add"] else 1)
        return {"bytes": T * D * (fs + (3 if case["residual"] else 2) * es) + 8 * T + D * ps + 2 * D * gs, "flops": 14 * T * D}
    if op in ("bias", "bias_grad"):
        table, seen = case["buckets"] * case["heads"] * ESIZE[case["param"]], _seen(case)
        if op == "bias":
            places = case["batch"] * case["heads"] * case["queries"] * case["keys"]
            return {"bytes": table + es * (places + (seen if case["add"] else 0)), "flops": seen * (2 if case["add"] else 1)}
        return {"bytes": table * (2 if case["add"] else 1) + es * seen, "flops": seen}
    T, E, k, ws = case["tokens"], case["experts"], case["chosen"], ESIZE[case["param"]]
    if op == "route":
        return {"bytes": T * (E * es + k * (4 + ws)) + 4 * E * (2 + case["replicas"]), "flops": T * E * (10 + k)}
    return {"bytes": T * (2 * E * es + k * (4 + ws)), "flops": T * E * 10}


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


def _normal(shape, dtype, seed, salt, sigma=1.0, mean=0.0):
    x = torch.empty(shape, dtype=TORCH[dtype], device="cuda")
    x.normal_(mean, sigma, generator=_gen(seed, salt))
    return x


def _rows(case, dtype, seed, salt, sigma=1.0, mean=0.0):
    return _normal((case["rows"], case["width"] + case["gap"]), dtype, seed, salt, sigma, mean)[:, :case["width"]]


def _norm_inputs(case, seed):
    st = _State()
    st.case = case
    D = case["width"]
    st.x = _rows(case, case["dtype"], seed, 1, 1.5, 0.3)
    st.residual = _rows(case, case["dtype"], seed, 2) if case["residual"] else None
    st.gamma = _normal((D,), case["param"], seed, 3, 0.1, 1.0)
    st.beta = _normal((D,), case["param"], seed, 4, 0.1)
    if case["op"] == "norm_grad":                 # residual: the gradient that flows back along the sum
        st.dy = _rows(case, case["flow"], seed, 5, 1e-2)
        st.dgamma = _normal((D,), case["grad"], seed, 6, 1e-2)
        st.dbeta = _normal((D,), case["grad"], seed, 7, 1e-2)
        if case["residual"]:
            st.residual.mul_(1e-2)
        mean, rstd = [], []
        for x in st.x.split(1 << 13):
            x = x.double()
            mean.append(x.mean(1))
            rstd.append(1.0 / (x.var(1, unbiased=False) + EPS).sqrt())
        st.mean, st.rstd = torch.cat(mean).float(), torch.cat(rstd).float()
    return st


def _lengths(case, of, seed, salt):
    if not case["ragged"]:
        return None
    u = torch.rand(case["batch"], generator=_gen(seed, salt), device="cuda", dtype=torch.float64)
    return (of - (u * (of // 2 + 1)).floor()).int()


def _bias_inputs(case, seed):
    st = _State()
    st.case = case
    B, H, Q, K = case["batch"], case["heads"], case["queries"], case["keys"]
    st.klen = _lengths(case, K, seed, 11)
    st.qlen = _lengths(case, Q, seed, 12) if case["op"] == "bias_grad" else None
    st.table = _normal((case["buckets"], H), case["param"], seed, 13, 0.5 if case["op"] == "bias" else 1e-2)
    shape = (B, H, Q, K + case["gap"])
    st.scores = None
    if case["op"] == "bias_grad" or case["add"]:
        st.scores = _normal(shape, case["dtype"], seed, 14, 1.0 if case["op"] == "bias" else 1e-3)[..., :K]
    return st


def _route_inputs(case, seed):
    st = _State()
    st.case = case
    T, E, k = case["tokens"], case["experts"], case["chosen"]
    st.logits = _normal((T, E + case["gap"]), case["dtype"], seed, 21, 1.5)[:, :E]
    if case["op"] == "route":
        st.bias = torch.randint(-40, 41, (E,), generator=_gen(seed, 22), device="cuda").float() * RATE
        R = max(1, case["replicas"])
        st.counts = torch.randint(0, 2 * T * k // E + 2, (R, E), generator=_gen(seed, 23), device="cuda", dtype=torch.int32)
    else:
        st.picked = torch.rand((T, E), generator=_gen(seed, 24), device="cuda").topk(k, dim=1).indices.int()
        st.dw = _normal((T, k), case["param"], seed, 25, 1e-2)
    return st


def prepare(case, seed):
    op = case["op"]
    if op in ("norm", "norm_grad"):
        st = _norm_inputs(case, seed)
        T, D, gap = case["rows"], case["width"], case["gap"]
        st.out = torch.zeros((T, D + gap), dtype=TORCH[case["dtype" if op == "norm_grad" else "flow"]], device="cuda")[:, :D]
        if op == "norm":
            st.total = torch.zeros((T, D + gap), dtype=TORCH[case["dtype"]], device="cuda")[:, :D] if case["residual"] else None
            st.mean = torch.zeros(T, device="cuda") if case["stats"] else None
            st.rstd = torch.zeros(T, device="cuda") if case["stats"] else None
    elif op in ("bias", "bias_grad"):
        st = _bias_inputs(case, seed)
        B, H, Q, K = case["batch"], case["heads"], case["queries"], case["keys"]
        if op == "bias":
            st.out = st.scores
            if st.out is None:
                st.out = torch.zeros((B, H, Q, K + case["gap"]), dtype=TORCH[case["dtype"]], device="cuda")[..., :K]
    else:
        st = _route_inputs(case, seed)
        T, E, k = case["tokens"], case["experts"], case["chosen"]
        if op == "route":
            st.picked = torch.zeros((T, k), dtype=torch.int32, device="cuda")
            st.weights = torch.zeros((T, k), dtype=TORCH[case["param"]], device="cuda")
            st.moved = torch.zeros(E, device="cuda")
        else:
            st.dlogits = torch.zeros((T, E + case["gap"]), dtype=TORCH[case["dtype"]], device="cuda")[:, :E]
    if own:
        import paper_2006_15704_amd as ddp
        stream = torch.cuda.current_stream().cuda_stream
        if op in ("norm", "norm_grad"):
            st.handle = ddp.ddp_layernorm_create(0, stream, case["width"])
            st.free = ddp.ddp_layernorm_destroy
        elif op in ("bias", "bias_grad"):
            st.handle = ddp.ddp_position_bias_create(0, stream, case["heads"], case["buckets"], case["exact"], case["distance"],
                                                     case["both"])
            st.free = ddp.ddp_position_bias_destroy
        else:
            st.handle = ddp.ddp_router_create(0, stream, case["experts"], case["chosen"], case["groups"], case["kept"], case["top"],
                                              case["score"], case["renorm"], case["scale"])
            st.free = ddp.ddp_router_destroy
    return st


# ---- passes ----

def run(st):
    op = st.case["op"]
    if own:
        import paper_2006_15704_amd as ddp
        return {"norm": _own_norm, "norm_grad": _own_norm_grad, "bias": _own_bias, "bias_grad": _own_bias_grad, "route": _own_route,
                "route_grad": _own_route_grad}[op](ddp, st)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "bias": _plain_bias, "bias_grad": _plain_bias_grad,
            "route": _plain_route, "route_grad": _plain_route_grad}[op](st)


def _at(x):
    return 0 if x is None else x.data_ptr()


def _step(x):
    return 0 if x is None else x.stride(0)


def _norm_outputs(st):
    out = {"y": st.out}
    if st.total is not None:
        out["sum"] = st.total
    if st.mean is not None:
        out["mean"], out["rstd"] = st.mean, st.rstd
    return out


def _own_norm(ddp, st):
    c = st.case
    ddp.ddp_layernorm_forward(st.handle, c["rows"], st.x.data_ptr(), c["dtype"], st.x.stride(0), _at(st.residual), _step(st.residual),
                              st.gamma.data_ptr(), st.beta.data_ptr(), c["param"], EPS, _at(st.total), _step(st.total),
                              st.out.data_ptr(), c["flow"], st.out.stride(0), _at(st.mean), _at(st.rstd))
    return _norm_outputs(st)


def _own_norm_grad(ddp, st):
    c = st.case
    ddp.ddp_layernorm_backward(st.handle, c["rows"], st.dy.data_ptr(), c["flow"], st.dy.stride(0), st.x.data_ptr(), c["dtype"],
                               st.x.stride(0), st.mean.data_ptr(), st.rstd.data_ptr(), st.gamma.data_ptr(), c["param"],
                               _at(st.residual), _step(st.residual), st.out.data_ptr(), st.out.stride(0), c["add"],
                               st.dgamma.data_ptr(), st.dbeta.data_ptr(), c["grad"])
    return {"dx": st.out, "dgamma": st.dgamma, "dbeta": st.dbeta}


def _own_bias(ddp, st):
    c, o = st.case, st.out
    ddp.ddp_position_bias_apply(st.handle, c["batch"], c["queries"], c["keys"], c["offset"], st.table.data_ptr(), c["param"],
                                st.table.stride(0), 1.0, _at(st.klen), c["causal"], LOWEST if c["dtype"] != 1 else -6e4, c["add"],
                                o.data_ptr(), c["dtype"], o.stride(0), o.stride(1), o.stride(2))
    return o


def _own_bias_grad(ddp, st):
    c, s = st.case, st.scores
    ddp.ddp_position_bias_grad(st.handle, c["batch"], c["queries"], c["keys"], c["offset"], s.data_ptr(), c["dtype"], s.stride(0),
                               s.stride(1), s.stride(2), 1.0, _at(st.klen), _at(st.qlen), c["causal"], c["add"],
                               st.table.data_ptr(), c["param"], st.table.stride(0))
    return st.table


def _own_route(ddp, st):
    c = st.case
    ddp.ddp_router_route(st.handle, c["tokens"], st.logits.data_ptr(), c["dtype"], st.logits.stride(0), st.bias.data_ptr(),
                         st.picked.data_ptr(), st.weights.data_ptr(), c["param"], st.counts.data_ptr(), False)
    if c["replicas"]:
        ddp.ddp_router_balance(st.handle, c["replicas"], st.counts.data_ptr(), RATE, st.bias.data_ptr(), st.moved.data_ptr())
    return _route_outputs(st)


def _route_outputs(st):
    out = {"experts": st.picked, "weights": st.weights, "counts": st.counts}
    if st.case["replicas"]:
        out["bias"] = st.moved
    return out


def _own_route_grad(ddp, st):
    c = st.case
    ddp.ddp_router_grad(st.handle, c["tokens"], st.logits.data_ptr(), c["dtype"], st.logits.stride(0), st.picked.data_ptr(),
                        st.dw.data_ptr(), c["param"], st.dlogits.data_ptr(), st.dlogits.stride(0))
    return st.dlogits


def _plain_norm(st):
    s = st.x.float()
    if st.residual is not None:
        s = s + st.residual.float()
        st.total.copy_(s)
    mean = s.mean(1, keepdim=True)
    s = s - mean
    rstd = 1.0 / ((s * s).mean(1, keepdim=True) + EPS).sqrt()
    st.out.copy_(s * rstd * st.gamma.float() + st.beta.float())
    if st.mean is not None:
        st.mean.copy_(mean[:, 0])
        st.rstd.copy_(rstd[:, 0])
    return _norm_outputs(st)


def _plain_norm_grad(st):
    dy = st.dy.float()
    xh = (st.x.float() - st.mean[:, None]) * st.rstd[:, None]
    g = dy * st.gamma.float()
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * st.rstd[:, None]
    if st.residual is not None:
        dx = dx + st.residual.float()
    st.out.copy_(dx)
    dgamma, dbeta = (dy * xh).sum(0, dtype=torch.float64), dy.sum(0, dtype=torch.float64)
    if st.case["add"]:
        dgamma, dbeta = dgamma + st.dgamma, dbeta + st.dbeta
    st.dgamma.copy_(dgamma)
    st.dbeta.copy_(dbeta)
    return {"dx": st.out, "dgamma": st.dgamma, "dbeta": st.dbeta}


def _first_distances(case):
    """The smallest distance of every bucket of one direction, in whole numbers (t steps of m: e (D / e)^(t / m))."""
    n, e, far = case["buckets"] // (2 if case["both"] else 1), case["exact"], case["distance"]
    m, first = n - e, list(range(e))
    for t in range(m):
        want = e ** (m - t) * far ** t if t else e ** m              # d^m >= this
        d = max(e, int(round(e * (far / e) ** (t / m))) - 2)
        while d ** m < want:
            d += 1
        first.append(d)
    return first


def _buckets_of(case, r):
    """Buckets of the relative positions r (keys minus queries)."""
    first = torch.tensor(_first_distances(case), device=r.device)
    if case["both"]:
        return torch.searchsorted(first, r.abs(), right=True) - 1 + (r > 0) * (case["buckets"] // 2)
    return torch.searchsorted(first, (-r).clamp(min=0), right=True) - 1


def _visible(case, klen, qlen):
    """(batch or 1, 1, queries, keys), or None: everything."""
    i, j = (torch.arange(case[w], device="cuda") for w in ("queries", "keys"))
    seen = None
    if case["causal"]:
        seen = (j[None, :] <= i[:, None] + case["offset"])[None, None]
    if klen is not None:
        here = (j[None, :] < klen[:, None])[:, None, None, :]
        seen = here if seen is None else seen & here
    if qlen is not None:
        here = (i[None, :] < qlen[:, None])[:, None, :, None]
        seen = here if seen is None else seen & here
    return seen


def _plain_bias(st):
    c = st.case
    Q, K = c["queries"], c["keys"]
    i, j = torch.arange(Q, device="cuda"), torch.arange(K, device="cuda")
    r = torch.arange(-(Q - 1) - c["offset"], K - c["offset"], device="cuda")
    of_distance = st.table.float()[_buckets_of(c, r)].t().contiguous()          # (heads, Q + K - 1)
    bias = of_distance[:, j[None, :] - i[:, None] + Q - 1][None]
    if c["add"]:
        bias = st.out.float() + bias
    seen = _visible(c, st.klen, None)
    if seen is not None:
        bias = torch.where(seen, bias, LOWEST if c["dtype"] != 1 else -6e4)
    st.out.copy_(bias)
    return st.out


def _plain_bias_grad(st):
    c = st.case
    Q, K, H = c["queries"], c["keys"], c["heads"]
    s = st.scores.float()
    seen = _visible(c, st.klen, st.qlen)
    if seen is not None:
        s = torch.where(seen, s, 0.0)
    s = s.sum(0).flip(1)                                                 # (heads, queries from the last, keys)
    # rows of Q + K places, read as rows of Q + K - 1: every row is one further to the right, so that a column is a diagonal
    s = torch.nn.functional.pad(s, (0, Q)).view(H, -1)[:, :Q * (Q + K - 1)].view(H, Q, Q + K - 1)
    s = s.sum(1, dtype=torch.float64)                                    # of r = -(Q - 1) - offset, ..., K - 1 - offset
    r = torch.arange(-(Q - 1) - c["offset"], K - c["offset"], device="cuda")
    grad = torch.zeros((c["buckets"], H), dtype=torch.float64, device="cuda")
    grad.index_add_(0, _buckets_of(c, r), s.t().contiguous())
    if c["add"]:
        grad = grad + st.table
    st.table.copy_(grad)
    return st.table


def _scores(case, logits):
    x = logits.double()
    return torch.softmax(x, 1) if case["score"] == 0 else torch.sigmoid(x)


def _plain_route(st):
    c = st.case
    T, E, k, G = c["tokens"], c["experts"], c["chosen"], c["groups"]
    s = _scores(c, st.logits)
    key = s + st.bias.double()
    if c["kept"] < G:
        best = key.view(T, G, E // G).sort(dim=2, descending=True).values[..., :min(c["top"], E // G)].sum(2)
        kept = best.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        open_ = torch.zeros((T, G), dtype=torch.bool, device="cuda").scatter_(1, kept, True)
        key = torch.where(open_.repeat_interleave(E // G, 1), key, -math.inf)
    picked = key.sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = s.gather(1, picked)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    st.picked.copy_(picked)
    st.weights.copy_(w * c["scale"])
    st.counts[0].copy_(torch.bincount(picked.reshape(-1), minlength=E))
    if c["replicas"]:
        count = st.counts.long().sum(0)
        st.moved.copy_(st.bias + RATE * torch.sign(count.sum() - count * E))
    return _route_outputs(st)


def _plain_route_grad(st):
    c = st.case
    s = _scores(c, st.logits).float()
    at = st.picked.long()
    dw, w = st.dw.float() * c["scale"], s.gather(1, at)
    if c["renorm"]:
        dw = (dw - (dw * w).sum(1, keepdim=True) / w.sum(1, keepdim=True)) / w.sum(1, keepdim=True)
    ds = torch.zeros_like(s).scatter_(1, at, dw)
    if c["score"] == 0:
        st.dlogits.copy_(s * (ds - (dw * w).sum(1, keepdim=True)))
    else:
        st.dlogits.copy_(ds * s * (1.0 - s))
    return st.dlogits


# ---- the same in 64 bits, from the definitions ----

def exact(case, seed):
    return {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "bias": _exact_bias, "bias_grad": _exact_bias_grad, "route": _exact_route,
            "route_grad": _exact_route_grad}[case["op"]](case, seed)


def _exact_norm(case, seed):
    st = _norm_inputs(case, seed)
    out = {"y": [], "sum": [], "mean": [], "rstd": []}
    gamma, beta = st.gamma.double(), st.beta.double()
    for a in range(0, case["rows"], 8192):
        s = st.x[a:a + 8192].double()
        if case["residual"]:
            s = s + st.residual[a:a + 8192].double()
        m = s.sum(1) / case["width"]
        v = ((s - m[:, None]) ** 2).sum(1) / case["width"]
        rstd = (v + EPS) ** -0.5
        out["y"].append(torch.addcmul(beta, (s - m[:, None]) * rstd[:, None], gamma))
        out["sum"].append(s)
        out["mean"].append(m)
        out["rstd"].append(rstd)
    keep = ["y"] + ["sum"] * case["residual"] + ["mean", "rstd"] * case["stats"]
    return {name: torch.cat(out[name]) for name in keep}


def _exact_norm_grad(case, seed):
    # the gradients of sum(dy * y) with mean and deviation as given: what they are of the row, the formula has eliminated
    st = _norm_inputs(case, seed)
    D = case["width"]
    dx = []
    dgamma = st.dgamma.double() * case["add"]
    dbeta = st.dbeta.double() * case["add"]
    for a in range(0, case["rows"], 8192):
        rows = slice(a, a + 8192)
        dy, mean, rstd = st.dy[rows].double(), st.mean[rows].double()[:, None], st.rstd[rows].double()[:, None]
        xh = st.x[rows].double().sub(mean).mul(rstd)
        dgamma += torch.sum(dy * xh, 0)
        dbeta += torch.sum(dy, 0)
        g = dy * st.gamma.double()
        inner = D * g - torch.sum(g, 1)[:, None] - xh * torch.sum(g * xh, 1)[:, None]
        d = inner * rstd / D
        dx.append(d + st.residual[rows].double() if case["residual"] else d)
    return {"dx": torch.cat(dx), "dgamma": dgamma, "dbeta": dbeta}


def _bucket(case, r):
    """Of one relative position, by trying the logarithm's steps one by one."""
    n = case["buckets"] // (2 if case["both"] else 1)
    side = n if case["both"] and r > 0 else 0
    d = abs(r) if case["both"] else max(-r, 0)
    e, far = case["exact"], case["distance"]
    if d < e:
        return side + d
    if d >= far or n == e:
        return side + n - 1
    t = 0
    while t + 1 < n - e and d ** (n - e) * e ** (t + 1) >= e ** (n - e) * far ** (t + 1):
        t += 1
    return side + min(e + t, n - 1)


def _bucket_rows(case):
    """The bucket of every place, (queries, keys)."""
    Q, K, o = case["queries"], case["keys"], case["offset"]
    of = torch.tensor([_bucket(case, r) for r in range(1 - Q - o, K - o)], device="cuda")
    return torch.stack([of[Q - 1 - i:Q - 1 - i + K] for i in range(Q)])


def _masked(case, st, b):
    """Places of sequence b that are not visible."""
    i = torch.arange(case["queries"], device="cuda")[:, None]
    j = torch.arange(case["keys"], device="cuda")[None, :]
    out = (j > i + case["offset"]) if case["causal"] else (j < 0) & (i < 0)
    if st.klen is not None:
        out = out | (j >= st.klen[b])
    if st.qlen is not None:
        out = out | (i >= st.qlen[b])
    return out


def _exact_bias(case, seed):
    st = _bias_inputs(case, seed)
    at, table = _bucket_rows(case), st.table.double()
    out = torch.zeros((case["batch"], case["heads"], case["queries"], case["keys"]), dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        hidden = _masked(case, st, b)
        for h in range(case["heads"]):
            v = torch.take(table[:, h].contiguous(), at)
            if case["add"]:
                v = v + st.scores[b, h].double()
            out[b, h] = v.masked_fill(hidden, LOWEST if case["dtype"] != 1 else -6e4)
    return out


def _exact_bias_grad(case, seed):
    st = _bias_inputs(case, seed)
    at = _bucket_rows(case)
    grad = st.table.double() * case["add"]
    for b in range(case["batch"]):
        seen = ~_masked(case, st, b)
        where = at[seen]
        order = where.argsort()
        count = torch.bincount(where, minlength=case["buckets"]).cumsum(0)
        for h in range(case["heads"]):
            run_ = torch.cat([torch.zeros(1, dtype=torch.float64, device="cuda"), st.scores[b, h][seen][order].double().cumsum(0)])
            upto = run_[count]
            grad[:, h] += torch.diff(upto, prepend=torch.zeros(1, dtype=torch.float64, device="cuda"))
    return grad


def _exact_route(case, seed):
    st = _route_inputs(case, seed)
    T, E, G = case["tokens"], case["experts"], case["groups"]
    x = st.logits.double()
    if case["score"] == 0:
        s = (x - x.amax(1, True)).exp()
        s = s / s.sum(1, True)
    else:
        s = 1.0 / (1.0 + (-x).exp())
    number = torch.arange(E, device="cuda").expand(T, E)
    key = s + st.bias.double()

    def largest(v, n):
        top = v.amax(1, True)
        return torch.where(v == top, n, 1 << 30).amin(1, True), top

    if case["kept"] < G:
        each = key.clone()
        rank = torch.zeros((T, G), dtype=torch.float64, device="cuda")
        for _ in range(min(case["top"], E // G)):
            for g in range(G):
                part = slice(g * (E // G), (g + 1) * (E // G))
                at, top = largest(each[:, part], number[:, part])
                rank[:, g] += top[:, 0]
                each.scatter_(1, at, -math.inf)
        allowed = torch.zeros((T, E), dtype=torch.bool, device="cuda")
        for _ in range(case["kept"]):
            at, _ = largest(rank, number[:, :G])
            rank.scatter_(1, at, -math.inf)
            allowed |= number // (E // G) == at
        key = key.masked_fill(~allowed, -math.inf)
    picked = []
    for _ in range(case["chosen"]):
        at, _ = largest(key, number)
        key.scatter_(1, at, -math.inf)
        picked.append(at)
    picked = torch.cat(picked, 1)
    w = torch.gather(s, 1, picked) * case["scale"]
    if case["renorm"]:
        w = w * case["scale"] / w.sum(1, True)
    counts = st.counts.clone()
    counts[0] = torch.stack([(picked == e).sum() for e in range(E)]).int()
    out = {"experts": picked.int(), "weights": w, "counts": counts}
    if case["replicas"]:
        load = counts.double().sum(0)
        out["bias"] = st.bias.double() + RATE * torch.sign(load.sum() / E - load)
    return out


def _exact_route_grad(case, seed):
    st = _route_inputs(case, seed)
    out = []
    for a in range(0, case["tokens"], 16384):
        rows = slice(a, a + 16384)
        x = st.logits[rows].double().requires_grad_()
        s = torch.softmax(x, 1) if case["score"] == 0 else torch.sigmoid(x)
        w = s.gather(1, st.picked[rows].long())
        if case["renorm"]:
            w = w / w.sum(1, True)
        out.append(torch.autograd.grad((w * case["scale"] * st.dw[rows].double()).sum(), x)[0])
    return torch.cat(out)
