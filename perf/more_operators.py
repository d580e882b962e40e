"""Performance cases of the feed-forward operators for batches of any length: a mixture of experts over tokens that are sorted
by expert, and 8-bit products with an epilogue.

  route     the experts of each token and their shares (`pick_experts`), and the pairs of tokens and experts sorted by expert
            (`sort_tokens`)
  gather    the tokens' rows in that order (`gather_tokens`)
  combine   the experts' rows back to their tokens, weighted and summed (`combine_tokens`)
  grad      the gradient of that (`combine_tokens_grad`)
  linear    residual + act(A W^T + bias) of 8-bit matrices (`linear_fp8`)
  experts   act(A W_e^T + bias_e) with each sorted row's own expert e (`experts_fp8`)

Pairs are numbered token by token.  `places[t, p]` is the row of pair (t, p) among the sorted ones, `tokens[row]` its token,
`offsets[e]` the first row of expert e and `offsets[E]` the number of rows that have an expert; pairs without one (id -1) come
behind.  An 8-bit matrix is e4m3 values with a scale per block of 1 x 128 (activations) or 128 x 128 (weights).

Where `own` is false the operators are computed with elementary torch operations in fp32; where it is true, by the package.
"""
import math

import torch

own = False

DEV = "cuda:0"
F8 = torch.float8_e4m3fn
BLOCK = 128
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def listed():
    """What the listed cases stand for:

    route_step       a decoding batch, 6 of 64 experts: latency
    route_many       a long prompt, 8 of 128 experts; a quarter of the logits is masked (experts of other groups)
    gather_ragged    fp32 rows of 3000 features with the shares applied; one pair in ten has no expert here
    gather_many      a long prompt's rows on their way into 8 large experts
    combine_token    one token's rows back from 6 experts, onto the residual: latency
    combine_many     a long prompt's rows back from 8 large experts, onto the residual
    grad_many        fine-tuning the router: the gradient of a prompt's sum over 8 of 64 experts
    linear_token     one token through a 9216 x 4096 layer with bias and GELU: the bytes of the weights
    linear_many      4096 tokens through a 4096 x 9216 layer with bias, onto the residual: matrix instructions
    experts_step     64 tokens, 2 of 8 experts of 4096 x 4096: the bytes of the weights
    experts_ragged   250 tokens, 4 of 16 experts of 1000 x 3000 with bias, SiLU and fp32 results: no size is a multiple of a tile
    experts_many     4096 tokens, 2 of 8 experts of 8192 x 4096: matrix instructions
    """
    return [
        {"op": "route", "T": 64, "E": 64, "P": 6, "x": "f32", "renormalise": True, "masked": 0.0, "name": "route_step"},
        {"op": "route", "T": 16384, "E": 128, "P": 8, "x": "bf16", "renormalise": False, "masked": 0.25, "name": "route_many"},
        {"op": "gather", "T": 330, "H": 3000, "P": 3, "E": 16, "x": "f32", "shares": True, "without": 0.1, "name": "gather_ragged"},
        {"op": "gather", "T": 8192, "H": 4096, "P": 2, "E": 8, "x": "bf16", "shares": False, "without": 0.0, "name": "gather_many"},
        {"op": "combine", "T": 1, "H": 2048, "P": 6, "E": 64, "x": "bf16", "shares": True, "residual": True, "without": 0.0,
         "name": "combine_token"},
        {"op": "combine", "T": 8192, "H": 4096, "P": 2, "E": 8, "x": "bf16", "shares": True, "residual": True, "without": 0.0,
         "name": "combine_many"},
        {"op": "grad", "T": 4096, "H": 2048, "P": 8, "E": 64, "x": "bf16", "without": 0.0, "name": "grad_many"},
        {"op": "linear", "M": 1, "N": 9216, "K": 4096, "out": "bf16", "bias": "f32", "act": "gelu", "residual": False, "name": "linear_token"},
        {"op": "linear", "M": 4096, "N": 4096, "K": 9216, "out": "bf16", "bias": "bf16", "act": "", "residual": True, "name": "linear_many"},
        {"op": "experts", "T": 64, "P": 2, "E": 8, "N": 4096, "K": 4096, "out": "bf16", "bias": "", "act": "", "sorted": False, "without": 0.0,
         "name": "experts_step"},
        {"op": "experts", "T": 250, "P": 4, "E": 16, "N": 1000, "K": 3000, "out": "f32", "bias": "f32", "act": "silu", "sorted": True,
         "without": 0.0, "name": "experts_ragged"},
        {"op": "experts", "T": 4096, "P": 2, "E": 8, "N": 8192, "K": 4096, "out": "bf16", "bias": "", "act": "", "sorted": False,
         "without": 0.0, "name": "experts_many"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A size between lo and hi: half of the time a multiple of 256."""
    n = _log(rng, lo, hi)
    return n // 256 * 256 if rng.random() < 0.5 and n >= 256 else n


def _experts(rng, most=256):
    """A number of experts: two thirds of the time a power of two."""
    n = _log(rng, 2, most)
    return 1 << (n.bit_length() - 1) if rng.random() < 0.67 else n


def draw(rng):
    """One more case of the same ranges: 1 to 16384 tokens (products: 8192), 1 to 8 of 2 to 256 experts, widths of 64 to 16384."""
    op = rng.choice(["route", "gather", "combine", "grad", "linear", "linear", "experts", "experts"])
    x = rng.choice(["bf16", "bf16", "f32"])
    without = rng.choice([0.0, 0.0, 0.2])
    if op == "route":
        E = _experts(rng)
        return {"op": op, "T": _log(rng, 1, 16384), "E": E, "P": rng.randint(1, min(8, E)), "x": x, "renormalise": rng.random() < 0.5,
                "masked": rng.choice([0.0, 0.25])}
    if op in ("gather", "combine", "grad"):
        E = _experts(rng)
        P, H = rng.randint(1, min(8, E)), _width(rng, 64, 9216)
        T = _log(rng, 1, max(1, min(8192, 2 ** 27 // (P * H * SIZE[x]))))
        case = {"op": op, "T": T, "H": H, "P": P, "E": E, "x": x, "without": without}
        if op != "grad":
            case["shares"] = rng.random() < 0.7
        if op == "combine":
            case["residual"] = rng.random() < 0.7
        return case
    act = rng.choice(["", "relu", "silu", "gelu", "gelu_tanh"])
    bias = rng.choice(["", "bf16", "f32"])
    out = rng.choice(["bf16", "bf16", "f32"])
    if op == "linear":
        N, K = _width(rng, 64, 16384), _width(rng, 64, 9216)
        M = _log(rng, 1, min(8192, max(1, 4096 * 4096 * 9216 // (N * K))))
        return {"op": op, "M": M, "N": N, "K": K, "out": out, "bias": bias, "act": act, "residual": rng.random() < 0.5}
    E = _experts(rng, 128)
    P, K = rng.randint(1, min(8, E)), _width(rng, 64, 4096)
    N = _width(rng, 64, max(128, min(8192, 8 * 8192 * 4096 // (E * K))))
    T = _log(rng, 1, max(1, min(8192, 4096 * 8192 * 4096 // (P * N * K))))
    return {"op": op, "T": T, "P": P, "E": E, "N": N, "K": K, "out": out, "bias": bias, "act": act, "sorted": rng.random() < 0.5,
            "without": without}


def _ceil(n, d):
    return -(-n // d)


def work(case):
    op = case["op"]
    if op == "route":
        T, E, P = case["T"], case["E"], case["P"]
        return {"bytes": T * E * SIZE[case["x"]] + 16 * T * P + 4 * (E + 1), "flops": 4 * T * E}
    if op in ("gather", "combine", "grad"):
        T, H, P, b = case["T"], case["H"], case["P"], SIZE[case["x"]]
        have = 1 - case["without"]  # pairs that have an expert
        plan = 4 * T * P * (2 if case.get("shares", op == "grad") else 1)
        if op == "gather":
            return {"bytes": T * H * b + T * P * H * b + plan, "flops": T * P * H if case["shares"] else 0}
        if op == "combine":
            return {"bytes": (have * P + 1 + case["residual"]) * T * H * b + plan, "flops": 2 * T * P * H}
        return {"bytes": (have * P + P + 1) * T * H * b + plan + 4 * T * P, "flops": 3 * T * P * H}
    N, K = case["N"], case["K"]
    kb = _ceil(K, BLOCK)
    weights = N * K + 4 * kb * _ceil(N, BLOCK) + N * SIZE.get(case["bias"], 0)
    if op == "linear":
        M = case["M"]
        return {"bytes": weights + M * (K + 4 * kb) + (1 + case["residual"]) * M * N * SIZE[case["out"]], "flops": 2 * M * N * K}
    T, P, E = case["T"], case["P"], case["E"]
    rows = T * P * (1 - case["without"])
    used = E * (1 - (1 - P / E) ** T)  # experts that some token picks, on average
    return {"bytes": used * weights + (rows if case["sorted"] else T) * (K + 4 * kb) + rows * N * SIZE[case["out"]] + 4 * T * P,
            "flops": 2 * rows * N * K}


# ---------------------------------------------------------------------------------------------- inputs

def _spread(s, rows, R, C):
    """The scale of each of R x C values."""
    s = s.repeat_interleave(BLOCK, -1)[..., :C]
    return s.repeat_interleave(rows, -2)[..., :R, :] if rows > 1 else s


def _quantise(y, rows):
    """fp32 values in 8 bits, with scales for blocks of rows x 128; rows on 16-byte boundaries."""
    R, C = y.shape[-2:]
    pad = torch.nn.functional.pad(y, (0, -C % BLOCK, 0, -R % rows))
    s = pad.abs().reshape(*y.shape[:-2], _ceil(R, rows), rows, _ceil(C, BLOCK), BLOCK).amax((-3, -1)).div(448).clamp(min=2.0 ** -126)
    del pad
    q = torch.zeros((*y.shape[:-1], _ceil(C, 16) * 16), dtype=torch.uint8, device=y.device)
    q[..., :C] = (y * _spread(1 / s, rows, R, C)).to(F8).view(torch.uint8)
    return q.view(F8)[..., :C], s


def _logits(normal, T, E):
    """Router logits: some experts are more popular than others, about by a factor of four."""
    return normal(T, E) + 0.35 * normal(1, E)


def _picks(case, normal, g):
    """ids [T, P] of different experts for each token, -1 for the pairs without one, and shares."""
    T, E, P = case["T"], case["E"], case["P"]
    best, ids = torch.sort(_logits(normal, T, E), dim=1, descending=True, stable=True)
    ids, shares = ids[:, :P].to(torch.int32), torch.softmax(best[:, :P], 1)
    if case["without"]:
        ids[torch.rand((T, P), generator=g, device=DEV) < case["without"]] = -1
    return ids.contiguous(), shares.contiguous()


def _sorted(ids, E):
    """places, tokens, offsets."""
    T, P = ids.shape
    flat = torch.where((ids < 0) | (ids >= E), E, ids).reshape(-1)
    order = torch.sort(flat, stable=True).indices
    places = torch.empty_like(order)
    places[order] = torch.arange(T * P, device=ids.device)
    counts = torch.zeros(E + 2, dtype=torch.int64, device=ids.device).index_add_(0, flat + 1, torch.ones_like(order))
    offsets = counts.cumsum(0)[:E + 1]
    return places.view(T, P).to(torch.int32), (order // P).to(torch.int32), offsets.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    s = dict(case)
    op = case["op"]
    if op == "route":
        logits = _logits(normal, case["T"], case["E"])
        if case["masked"]:
            logits[torch.rand(logits.shape, generator=g, device=DEV) < case["masked"]] = -math.inf
        s["logits"] = logits.to(TYPES[case["x"]])
        return s
    if op in ("gather", "combine", "grad"):
        T, H, P, t = case["T"], case["H"], case["P"], TYPES[case["x"]]
        ids, shares = _picks(case, normal, g)
        s["places"], _, s["offsets"] = _sorted(ids, case["E"])
        s["shares"] = shares if case.get("shares", True) else None
        if op != "combine":
            s["X"] = normal(T, H).to(t)
        if op != "gather":
            s["R"] = normal(T * P, H).to(t)
        if op == "combine":
            s["residual"] = (4 * normal(T, H)).to(t) if case["residual"] else None
        return s
    N, K, t = case["N"], case["K"], TYPES[case["out"]]
    if op == "linear":
        M = case["M"]
        s["A"], sa = _quantise(normal(M, K) * torch.exp(normal(1, K)), 1)
        s["W"], s["SW"] = _quantise(normal(N, K) / math.sqrt(K), BLOCK)
        s["b"] = normal(N).to(TYPES[case["bias"]]) if case["bias"] else None
        s["r"] = (4 * normal(M, N)).to(t) if case["residual"] else None
    else:
        T, P, E = case["T"], case["P"], case["E"]
        ids, _ = _picks(case, normal, g)
        _, s["tokens"], s["offsets"] = _sorted(ids, E)
        s["A"], sa = _quantise(normal(T * P if case["sorted"] else T, K) * torch.exp(normal(1, K)), 1)
        s["W"], s["SW"] = _quantise(normal(E, N, K) / math.sqrt(K), BLOCK)
        s["b"] = normal(E, N).to(TYPES[case["bias"]]) if case["bias"] else None
        s["Y"] = torch.zeros((T * P, N), dtype=t, device=DEV)  # what rows without an expert keep
        s["longest"] = int(s["offsets"].diff().max())
    s["SA"] = sa.t().contiguous().t()  # block column by block column, as the package's operators write it
    return s


# ---------------------------------------------------------------------------------------------- the operators

def _act(name, x):
    if name == "relu":
        return torch.where(x < 0, 0.0, x)
    if name == "silu":
        return x / (1 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return x / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return x


def _dense(q, s, rows):
    return q.float() * _spread(s, rows, *q.shape[-2:])


def _plain(s):
    op = s["op"]
    if op == "route":
        logits, P = s["logits"].float(), s["P"]
        best, ids = torch.sort(logits, dim=1, descending=True, stable=True)
        some = best[:, :1] > -math.inf
        e = torch.where(some, torch.exp(best - torch.where(some, best[:, :1], 0.0)), 0.0)
        total = (e[:, :P] if s["renormalise"] else e).sum(1, keepdim=True)
        shares = torch.where(some, e[:, :P] / total, 0.0)
        ids = torch.where(best[:, :P] > -math.inf, ids[:, :P], -1).to(torch.int32)
        return (ids, shares, *_sorted(ids, s["E"]))
    if op in ("gather", "combine", "grad"):
        places = s["places"].long()
        have = (s["places"] < s["offsets"][-1]).unsqueeze(2)
    if op == "gather":
        x = s["X"].float().unsqueeze(1)
        x = x * s["shares"].unsqueeze(2) if s["shares"] is not None else x.expand(-1, s["P"], -1)
        out = torch.empty((s["T"] * s["P"], s["H"]), dtype=s["X"].dtype, device=x.device)
        out[places] = torch.where(have, x, 0.0).to(out.dtype)
        return out
    if op == "combine":
        r = s["R"][places].float()
        r = r if s["shares"] is None else r * s["shares"].unsqueeze(2)
        y = torch.where(have, r, 0.0).sum(1)
        return (y if s["residual"] is None else y + s["residual"].float()).to(s["R"].dtype)
    if op == "grad":
        dy = s["X"].float().unsqueeze(1)
        dshares = torch.where(have, s["R"][places].float() * dy, 0.0).sum(2)
        dR = torch.empty_like(s["R"])
        dR[places] = torch.where(have, dy * s["shares"].unsqueeze(2), 0.0).to(dR.dtype)
        return dR, dshares
    b = None if s["b"] is None else s["b"].float()
    if op == "linear":
        y = _dense(s["A"], s["SA"], 1) @ _dense(s["W"], s["SW"], BLOCK).t()
        y = _act(s["act"], y if b is None else y + b)
        return (y if s["r"] is None else y + s["r"].float()).to(TYPES[s["out"]])
    # every expert's rows in a batch as long as the longest needs
    offsets, a = s["offsets"].long(), _dense(s["A"], s["SA"], 1)
    at = offsets[:-1, None] + torch.arange(s["longest"], device=a.device)
    there = at < offsets[1:, None]
    first = torch.where(there, at, 0)
    a = a[first] if s["sorted"] else a[s["tokens"].long()[first]]
    y = a @ _dense(s["W"], s["SW"], BLOCK).transpose(1, 2)
    y = _act(s["act"], y if b is None else y + b.unsqueeze(1)).to(TYPES[s["out"]])
    R, N = s["Y"].shape
    out = torch.empty((R + 1, N), dtype=s["Y"].dtype, device=a.device)
    out[:R] = s["Y"]
    out[torch.where(there, at, R)] = y  # what is no row goes behind the last
    return out[:R]


def _own(s):
    import paper_1905_10138_amd as xe
    op = s["op"]
    if op == "route":
        ids, shares = xe.pick_experts(s["logits"], s["P"], renormalise=s["renormalise"])
        return (ids, shares, *xe.sort_tokens(ids, s["E"]))
    if op == "gather":
        return xe.gather_tokens(s["X"], s["places"], s["offsets"], s["shares"])
    if op == "combine":
        return xe.combine_tokens(s["R"], s["places"], s["offsets"], s["shares"], s["residual"])
    if op == "grad":
        return xe.combine_tokens_grad(s["X"], s["R"], s["places"], s["offsets"], s["shares"])
    if op == "linear":
        return xe.linear_fp8(s["A"], s["SA"], s["W"], s["SW"], bias=s["b"], activation=s["act"] or None, residual=s["r"], out_dtype=TYPES[s["out"]])
    return xe.experts_fp8(s["A"], s["SA"], s["W"], s["SW"], s["offsets"], tokens=None if s["sorted"] else s["tokens"], bias=s["b"],
                          activation=s["act"] or None, Y=s["Y"])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------- in 64 bits

def _values(q, s, rows):
    """What an 8-bit matrix stands for."""
    r = torch.arange(q.shape[0], device=q.device) // rows
    c = torch.arange(q.shape[1], device=q.device) // BLOCK
    return q.double() * s.double()[r][:, c]


def _exact_act(name, x):
    if name == "relu":
        return x.clamp(min=0)
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return x * torch.special.ndtr(x)
    if name == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    return x


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        T, E, P = case["T"], case["E"], case["P"]
        logits = s["logits"].double()
        left, index = logits.clone(), torch.arange(E, device=DEV)
        ids = torch.empty((T, P), dtype=torch.int64, device=DEV)
        for p in range(P):  # the largest that is left, the first of equals
            most = left.amax(1, keepdim=True)
            ids[:, p] = torch.where(left == most, index, E).amin(1)
            ids[:, p].masked_fill_(most[:, 0] == -math.inf, -1)
            left.scatter_(1, ids[:, p:p + 1].clamp(min=0), -math.inf)
        picked = torch.where(ids < 0, -math.inf, logits.gather(1, ids.clamp(min=0)))
        total = torch.logsumexp(picked if case["renormalise"] else logits, 1, keepdim=True)
        shares = torch.where(ids < 0, 0.0, torch.exp(picked - torch.where(total > -math.inf, total, 0.0)))
        flat = ids.reshape(-1)
        key = torch.where(flat < 0, E, flat) * (T * P) + torch.arange(T * P, device=DEV)
        key = torch.sort(key).values  # all different: by expert, then by pair
        pairs, places = key % (T * P), torch.empty_like(key)
        places.scatter_(0, pairs, torch.arange(T * P, device=DEV))
        offsets = torch.searchsorted(key, torch.arange(E + 1, device=DEV) * (T * P))
        return ids.to(torch.int32), shares, places.view(T, P).to(torch.int32), (pairs // P).to(torch.int32), offsets.to(torch.int32)
    if op in ("gather", "combine", "grad"):
        T, H, P = case["T"], case["H"], case["P"]
        rows = int(s["offsets"][-1])
        pair_of = torch.empty(T * P, dtype=torch.int64, device=DEV)
        pair_of[s["places"].reshape(-1).long()] = torch.arange(T * P, device=DEV)
        pair = pair_of[:rows]  # of each row
        share = torch.ones(T * P, device=DEV) if s["shares"] is None else s["shares"].reshape(-1)
        share = share.double()[pair].unsqueeze(1)
        if op == "gather":
            out = torch.zeros((T * P, H), dtype=torch.float64, device=DEV)
            out[:rows] = s["X"].double()[pair // P] * share
            return out
        if op == "combine":
            y = torch.zeros((T, H), dtype=torch.float64, device=DEV) if s["residual"] is None else s["residual"].double()
            return y.index_add(0, pair // P, s["R"][:rows].double() * share)
        dy = s["X"].double()[pair // P]
        dR, dshares = torch.zeros((T * P, H), dtype=torch.float64, device=DEV), torch.zeros(T * P, dtype=torch.float64, device=DEV)
        dR[:rows] = dy * share
        dshares[pair] = torch.linalg.vecdot(dy, s["R"][:rows].double())
        return dR, dshares.view(T, P)
    if op == "linear":
        y = torch.mm(_values(s["A"], s["SA"], 1), _values(s["W"], s["SW"], BLOCK).t())
        y = _exact_act(case["act"], y if s["b"] is None else y + s["b"].double())
        return y if s["r"] is None else y + s["r"].double()
    y = torch.zeros((case["T"] * case["P"], case["N"]), dtype=torch.float64, device=DEV)
    a = _values(s["A"], s["SA"], 1)
    a = a if case["sorted"] else a[s["tokens"].long()]
    offsets = s["offsets"].tolist()
    for e in range(case["E"]):
        here = slice(offsets[e], offsets[e + 1])
        if offsets[e] < offsets[e + 1]:
            z = torch.mm(a[here], _values(s["W"][e], s["SW"][e], BLOCK).t())
            y[here] = _exact_act(case["act"], z if s["b"] is None else z + s["b"][e].double())
    return y
