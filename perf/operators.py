"""The dense products of the feed-forward blocks that stay unfolded, as cases that can be timed and compared.

``tardis_linear``            y = act(x W^T + b) + r: a dense FFN's two products, a projection, router logits
``tardis_route``             the experts of every token: top-k of the router's logits, weights, rows sorted by expert
``tardis_grouped_linear``    the same product with the weights of each row's expert, rows grouped by expert, sizes ragged
``tardis_grouped_linear_combine``   the second product of the experts' FFNs and the weighted sum back to the tokens

``listed()`` names cases from one token of a decoding step to prompts; ``draw()`` gives others of the same ranges.
Weights and tokens are seeded stand-ins with the structure of ``workloads/generate.py``: weights N(0, 0.02^2), biases
N(0, 0.01^2), layer-normalised heavy-tailed tokens; inputs of second products are GELU outputs.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- the cases --------------------------------------------------------------------------------------------------
def _linear(n, k, o, act="none", bias=True, residual=False, dtype="bf16", out="same"):
    """x [n, k] times W [o, k]."""
    return dict(kind="linear", n=n, k=k, o=o, act=act, bias=bias, residual=residual, dtype=dtype, out=dtype if out == "same" else out)


def _route(tokens, experts, top_k, normalise=True, padded=0.0):
    """padded: the share of the tokens, at the end of the batch, that are masked for every expert."""
    return dict(kind="route", tokens=tokens, experts=experts, top_k=top_k, normalise=normalise, padded=padded)


def _up(tokens, experts, top_k, k, o, act="tanh", bias=True, skew=0.5, padded=0.0, dtype="bf16"):
    """The experts' first product: rows of x gathered by expert."""
    return dict(kind="up", tokens=tokens, experts=experts, top_k=top_k, k=k, o=o, act=act, bias=bias, skew=skew, padded=padded, dtype=dtype)


def _down(tokens, experts, top_k, k, o, bias=True, residual=True, skew=0.5, padded=0.0, dtype="bf16"):
    """The experts' second product and the weighted sum back to the tokens."""
    return dict(kind="down", tokens=tokens, experts=experts, top_k=top_k, k=k, o=o, bias=bias, residual=residual, skew=skew, padded=padded,
                dtype=dtype)


def listed():
    return [
        # one decoding step of one sequence, first product of a dense 4096 / 16384 layer
        dict(_linear(1, 4096, 16384, act="tanh"), name="linear_up_1_token"),
        # four sequences, second product of a dense 4544 / 18176 layer, added to the residual stream
        dict(_linear(4, 18176, 4544, residual=True), name="linear_down_4_tokens"),
        # continuous batching of 64 sequences, second product with residual
        dict(_linear(64, 16384, 4096, residual=True), name="linear_down_64_tokens"),
        # a ragged prompt through the first product of a 4544 / 18176 layer with the erf form
        dict(_linear(777, 4544, 18176, act="erf"), name="linear_up_777_tokens"),
        # prompts: 8 sequences of 2048 tokens
        dict(_linear(16384, 4096, 16384, act="tanh"), name="linear_up_16384_tokens"),
        # the small fp32 layer
        dict(_linear(64, 256, 1024, act="relu", residual=True, dtype="f32"), name="linear_f32_64_tokens"),
        # routing of a decoding step and of prompts whose last eighth is padding
        dict(_route(4, 8, 2), name="route_4_tokens"),
        dict(_route(16384, 64, 4, normalise=False, padded=0.125), name="route_16384_tokens"),
        # experts' FFNs: one token; a prompt
        dict(_up(1, 8, 2, 4096, 16384), name="experts_up_1_token"),
        dict(_up(4096, 8, 2, 4096, 16384), name="experts_up_4096_tokens"),
        # many small experts, 48 sequences in a decoding step; a ragged prompt
        dict(_down(48, 64, 4, 4096, 1024), name="experts_down_48_tokens"),
        dict(_down(2000, 16, 2, 8192, 2048, skew=1.0, padded=0.05), name="experts_down_2000_tokens"),
    ]


def _log_int(rng, lo, hi, multiple=1):
    """A whole number, spread evenly over the logarithm of [lo, hi], rounded to the multiple."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / multiple)) * multiple))


MOST_FLOPS = 2.0 * 16384 * 4096 * 16384
MOST_WEIGHTS = 2 ** 29          # elements of all weights of a case


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "route", "up", "up", "down", "down"])
    if kind == "route":
        experts = _log_int(rng, 2, 256)
        return _route(_log_int(rng, 1, 16384), experts, rng.randint(1, min(8, experts)), normalise=rng.random() < 0.5,
                      padded=rng.choice([0.0, 0.0, 0.1, 0.6]))
    small = rng.random() < 0.15                     # fp32 layers are small ones
    dtype = "f32" if small else "bf16"
    k = _log_int(rng, 64, 1024 if small else 18176, 8)
    o = _log_int(rng, 8, 2048 if small else 18176)
    act = rng.choice(["none", "tanh", "erf", "relu"])
    bias, residual = rng.random() < 0.7, rng.random() < 0.5
    if kind == "linear":
        n = _log_int(rng, 1, 2048 if small else 16384)
        n = max(1, min(n, int(MOST_FLOPS / (2.0 * k * o))))
        return _linear(n, k, o, act=act, bias=bias, residual=residual, dtype=dtype, out=rng.choice([dtype, dtype, "f32"]))
    experts = _log_int(rng, 2, 128)
    top_k = rng.randint(1, min(8, experts))
    while experts * k * o > MOST_WEIGHTS:           # smaller experts where there are many
        if k >= o:
            k = max(64, k // 16 * 8)
        else:
            o = max(8, o // 2)
    tokens = _log_int(rng, 1, 1024 if small else 8192)
    tokens = max(1, min(tokens, int(MOST_FLOPS / (2.0 * k * o * top_k)), 32768 // top_k))
    skew, padded = rng.choice([0.0, 0.5, 1.0, 2.0]), rng.choice([0.0, 0.0, 0.1, 0.6])
    if kind == "up":
        return _up(tokens, experts, top_k, k, o, act=act, bias=bias, skew=skew, padded=padded, dtype=dtype)
    return _down(tokens, experts, top_k, k, o, bias=bias, residual=residual, skew=skew, padded=padded, dtype=dtype)


# ---- inputs -----------------------------------------------------------------------------------------------------
def _tokens(n, d, g):
    z = torch.randn(n, d, generator=g, device=DEVICE)
    v = torch.zeros(n, d, device=DEVICE)
    for _ in range(4):                              # chi-square with 4 degrees of freedom: Student-t tokens
        v += torch.randn(n, d, generator=g, device=DEVICE) ** 2
    x = z / torch.sqrt(v / 4)
    x -= x.mean(dim=-1, keepdim=True)
    return x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + 1e-5)


def _hidden(n, d, g):
    """GELU outputs of pre-activations with deviation 1.28 (weights of 0.02 on 4096 normalised channels)."""
    z = torch.randn(n, d, generator=g, device=DEVICE) * 1.28
    return 0.5 * z * (1 + torch.tanh(0.7978845608028654 * (z + 0.044715 * z ** 3)))


def _logits(case, g):
    t, e = case["tokens"], case["experts"]
    logits = torch.randn(t, e, generator=g, device=DEVICE) + case.get("skew", 0.5) * torch.randn(1, e, generator=g, device=DEVICE)
    kept = t - int(t * case["padded"])
    logits[max(1, kept):] = -math.inf
    return logits


def _weights(shape, g, dtype):
    return (torch.randn(*shape, generator=g, device=DEVICE) * 0.02).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    state = dict(case=case)
    if case["kind"] == "route":
        state["logits"] = _logits(case, g)
        return state
    dtype, k, o = DTYPES[case["dtype"]], case["k"], case["o"]
    if case["kind"] == "linear":
        made = _hidden if k > o else _tokens
        state["x"] = made(case["n"], k, g).to(dtype)
        state["W"] = _weights((o, k), g, dtype)
        state["b"] = torch.randn(o, generator=g, device=DEVICE) * 0.01 if case["bias"] else None
        state["r"] = torch.randn(case["n"], o, generator=g, device=DEVICE).to(DTYPES[case["out"]]) if case["residual"] else None
        return state
    experts, top_k = case["experts"], case["top_k"]
    _, state["weights"], state["offsets"], state["rows"], state["slots"] = _plain_route(_logits(case, g), top_k, True)
    state["W"] = torch.empty(experts, o, k, dtype=dtype, device=DEVICE)
    for e in range(experts):
        state["W"][e] = _weights((o, k), g, dtype)
    state["b"] = torch.randn(experts, o, generator=g, device=DEVICE) * 0.01 if case["bias"] else None
    if case["kind"] == "up":
        state["x"] = _tokens(case["tokens"], k, g).to(dtype)
        state["y"] = torch.zeros(case["tokens"] * top_k, o, dtype=dtype, device=DEVICE)      # rows behind the last group stay zero
    else:
        state["x"] = _hidden(case["tokens"] * top_k, k, g).to(dtype)
        state["r"] = torch.randn(case["tokens"], o, generator=g, device=DEVICE).to(dtype) if case["residual"] else None
    return state


# ---- one pass ---------------------------------------------------------------------------------------------------
def _act(z, act):
    if act == "tanh":
        return 0.5 * z * (1 + torch.tanh(0.7978845608028654 * (z + 0.044715 * z * z * z)))
    if act == "erf":
        return 0.5 * z * (1 + torch.erf(z * 0.7071067811865476))
    return torch.clamp(z, min=0) if act == "relu" else z


def _plain_route(logits, top_k, normalise):
    t, e = logits.shape
    dev = logits.device
    l = torch.where(torch.isnan(logits), torch.full_like(logits, -math.inf), logits)
    top, chosen = torch.sort(l, dim=1, descending=True, stable=True)       # equal logits: the lowest expert first
    biggest = top[:, :1]
    none = top[:, :top_k] == -math.inf
    share = torch.exp(torch.where(top == biggest, torch.zeros_like(top), top - biggest))
    share = torch.where(top == -math.inf, torch.zeros_like(share), share)
    total = (share[:, :top_k] if normalise else share).sum(dim=1, keepdim=True)
    weights = torch.where(none, torch.zeros_like(share[:, :top_k]), share[:, :top_k] / total)
    chosen = torch.where(none, torch.full_like(chosen[:, :top_k], e), chosen[:, :top_k])
    order = torch.argsort(chosen.reshape(-1), stable=True)                 # by expert, then by token
    by_expert = chosen.reshape(-1)[order]
    offsets = torch.searchsorted(by_expert, torch.arange(e + 1, device=dev))
    rows = torch.where(by_expert < e, torch.div(order, top_k, rounding_mode="floor"), torch.full_like(order, -1))
    slots = torch.empty_like(order)
    slots[order] = torch.where(by_expert < e, torch.arange(t * top_k, device=dev), torch.full_like(order, -1))
    experts = torch.where(none, torch.full_like(chosen, -1), chosen)
    return experts.int(), weights, offsets.int(), rows.int(), slots.reshape(t, top_k).int()


def _plain_groups(state, x, act):
    """act(W_e x + b_e) of every row, in 32 bits; rows behind the last group are zero."""
    W, b = state["W"], state["b"]
    z = torch.zeros(x.shape[0], W.shape[1], dtype=torch.float32, device=x.device)
    ends = state["offsets"].tolist()
    for e in range(W.shape[0]):
        lo, hi = ends[e], ends[e + 1]
        if hi > lo:
            part = x[lo:hi].float() @ W[e].float().T
            z[lo:hi] = _act(part + b[e] if b is not None else part, act)
    return z


def _plain(state):
    case = state["case"]
    if case["kind"] == "route":
        return _plain_route(state["logits"], case["top_k"], case["normalise"])
    if case["kind"] == "linear":
        z = state["x"].float() @ state["W"].float().T
        if state["b"] is not None:
            z = z + state["b"]
        z = _act(z, case["act"])
        if state["r"] is not None:
            z = z + state["r"].float()
        return z.to(DTYPES[case["out"]])
    if case["kind"] == "up":
        rows = state["rows"].long().clamp(min=0)
        return _plain_groups(state, state["x"][rows], case["act"]).to(DTYPES[case["dtype"]])
    f = _plain_groups(state, state["x"], "none")
    slots = state["slots"].long()
    part = torch.where(slots[:, :, None] >= 0, f[slots.clamp(min=0)] * state["weights"][:, :, None], torch.zeros((), device=f.device))
    y = part.sum(dim=1)
    if state["r"] is not None:
        y = y + state["r"].float()
    return y.to(DTYPES[case["dtype"]])


def run(state):
    if not own:
        return _plain(state)
    import paper_2501_10054_b200 as T
    case = state["case"]
    act = {"none": T.TARDIS_ACT_NONE, "tanh": T.TARDIS_ACT_GELU_TANH, "erf": T.TARDIS_ACT_GELU_ERF,
           "relu": T.TARDIS_ACT_RELU}[case.get("act", "none")]
    if case["kind"] == "route":
        return T.tardis_route(state["logits"], case["top_k"], normalise=case["normalise"])
    if case["kind"] == "linear":
        return T.tardis_linear(state["x"], state["W"], bias=state["b"], act=act, residual=state["r"], out_dtype=DTYPES[case["out"]])
    if case["kind"] == "up":
        return T.tardis_grouped_linear(state["x"], state["W"], state["offsets"], bias=state["b"], act=act, rows=state["rows"],
                                       out=state["y"])
    return T.tardis_grouped_linear_combine(state["x"], state["W"], state["offsets"], state["slots"], state["weights"], bias=state["b"],
                                           residual=state["r"])


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "route":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        return {"bytes": 4.0 * (t * e + 4 * t * k + e + 1), "flops": 5.0 * t * e}
    size, k, o = DTYPES[case["dtype"]].itemsize, case["k"], case["o"]
    if case["kind"] == "linear":
        n, out = case["n"], DTYPES[case["out"]].itemsize
        moved = size * (n * k + o * k) + out * n * o * (2 if case["residual"] else 1) + (4 * o if case["bias"] else 0)
        return {"bytes": float(moved), "flops": 2.0 * n * k * o}
    # experts with rows: as many as tokens that choose evenly would reach
    t = case["tokens"] - min(case["tokens"] - 1, int(case["tokens"] * case["padded"]))
    rows, experts = t * case["top_k"], case["experts"]
    reached = experts * (1.0 - (1.0 - case["top_k"] / experts) ** t)
    weights = reached * (size * o * k + (4 * o if case["bias"] else 0))
    if case["kind"] == "up":
        moved = weights + size * (t * k + rows * o) + 4 * (rows + experts + 1)
    else:
        moved = weights + size * (rows * k + case["tokens"] * o * (2 if case["residual"] else 1)) + 8 * rows + 4 * (experts + 1)
    return {"bytes": float(moved), "flops": 2.0 * rows * k * o}


# ---- the definitions, in 64 bits --------------------------------------------------------------------------------
def _exact_act(z, act):
    if act == "tanh":
        return z / (1 + torch.exp(-1.5957691216057308 * (z + 0.044715 * z ** 3)))
    if act == "erf":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    return torch.where(z > 0, z, torch.zeros_like(z)) if act == "relu" else z


def _exact_route(logits, top_k, normalise):
    """The k largest by k rounds of taking the largest; places by counting the tokens before."""
    t, e = logits.shape
    dev, index = logits.device, torch.arange(e, device=logits.device)
    left = torch.nan_to_num(logits.double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    top = left.max(dim=1, keepdim=True).values
    share = torch.where(left == top, 1.0, torch.exp(left - top)).masked_fill(left == -math.inf, 0.0)
    experts = torch.full((t, top_k), -1, dtype=torch.int64, device=dev)
    weights = torch.zeros(t, top_k, dtype=torch.float64, device=dev)
    member = torch.zeros(t, e, dtype=torch.int64, device=dev)
    for j in range(top_k):
        best = left.max(dim=1, keepdim=True).values
        pick = torch.where(left == best, index, e).min(dim=1, keepdim=True).values
        ok = best > -math.inf
        experts[:, j:j + 1] = torch.where(ok, pick, -1)
        weights[:, j:j + 1] = torch.where(ok, share.gather(1, pick), 0.0)
        member.scatter_add_(1, pick, ok.long())
        left.scatter_(1, pick, -math.inf)
    total = weights.sum(dim=1, keepdim=True) if normalise else share.sum(dim=1, keepdim=True)
    weights = torch.where(experts >= 0, weights / total, 0.0)
    offsets = torch.zeros(e + 1, dtype=torch.int64, device=dev)
    offsets[1:] = member.sum(dim=0).cumsum(0)
    place = offsets[:-1] + member.cumsum(0) - member
    slots = torch.where(experts >= 0, place.gather(1, experts.clamp(min=0)), -1)
    rows = torch.full((t * top_k + 1,), -1, dtype=torch.int64, device=dev)
    token = torch.arange(t, device=dev)[:, None].expand(t, top_k)
    rows.scatter_(0, torch.where(slots >= 0, slots, t * top_k).reshape(-1), token.reshape(-1))
    return experts.int(), weights, offsets.int(), rows[:-1].int(), slots.int()


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "route":
        return _exact_route(state["logits"], case["top_k"], case["normalise"])
    x, W, b = state["x"].double(), state["W"], state["b"]
    if case["kind"] == "linear":
        z = torch.nn.functional.linear(x, W.double(), None if b is None else b.double())
        y = _exact_act(z, case["act"])
        return y if state["r"] is None else y + state["r"].double()
    offsets = state["offsets"].cpu().numpy()
    if case["kind"] == "up":
        x = x.index_select(0, state["rows"].long().clamp(min=0))
    f = torch.zeros(x.shape[0], case["o"], dtype=torch.float64, device=x.device)
    for e in range(case["experts"]):
        own_rows = slice(int(offsets[e]), int(offsets[e + 1]))
        f[own_rows] = torch.einsum("rk,ok->ro", x[own_rows], W[e].double())
        if b is not None:
            f[own_rows] += b[e].double()
        f[own_rows] = _exact_act(f[own_rows], case.get("act", "none"))
    if case["kind"] == "up":
        return f
    y = torch.zeros(case["tokens"], case["o"], dtype=torch.float64, device=x.device)
    for j in range(case["top_k"]):
        slot = state["slots"][:, j].long()
        there = slot >= 0
        y[there] += state["weights"][there, j, None].double() * f[slot[there]]
    return y if state["r"] is None else y + state["r"].double()
