"""tardis_linear, tardis_grouped_linear (plain and with the return to the tokens) and tardis_route against their definitions in
64 bits on the same inputs.

The bound of a sum of k products in fp32: bf16 products are exact, the tensor cores add at least 8 of them (half of an instruction's
16 channels) before they round or cut off to 24 bits, so at most k / 8 + 16 partial sums lose 2^-23 of a value that is at most
S = sum |x w| (16 covers the joining of split channel ranges); for fp32 outputs an accumulator takes 512 channels at most and the parts
are rounded to nearest, k / 512 of them; plain fp32 multiply-adds round k times by 2^-24.  The activations' slopes
are below 1.13; evaluating one in fp32 costs a few roundings of |z|.  Bias and residual: one rounding each.  Then the output's own."""
import math

import numpy as np
import pytest
import torch

import paper_2501_10054_b200 as T

gpu = pytest.mark.gpu
NONE, TANH, ERF, RELU = T.TARDIS_ACT_NONE, T.TARDIS_ACT_GELU_TANH, T.TARDIS_ACT_GELU_ERF, T.TARDIS_ACT_RELU
BF, F32 = torch.bfloat16, torch.float32


def act64(z, act):
    if act == TANH:
        return z / (1 + torch.exp(-1.5957691216057308 * (z + 0.044715 * z ** 3)))
    if act == ERF:
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    return torch.clamp(z, min=0) if act == RELU else z


def product64(x, W, bias, act, out=None):
    """f and the bound of its error, both float64 (see the head of the file)."""
    k = x.shape[1]
    z = x.double() @ W.double().T
    mag = x.double().abs() @ W.double().abs().T
    if bias is not None:
        z = z + bias.double()
        mag = mag + bias.double().abs()
    steps = (k + 2) * 2.0 ** -24
    if x.dtype == BF:
        steps = (k / 8 + 16 if out != F32 else min(k, 512) / 8 + k / 1024 + 16) * 2.0 ** -23
    tol = 1.13 * steps * mag + (8 * 2.0 ** -24 * z.abs() if act != NONE else 0)
    return act64(z, act), tol


def check(got, ref, tol, residual=None):
    """tol: bound in front of the residual and the output's rounding."""
    if residual is not None:
        ref = ref + residual.double()
        tol = tol + 2.0 ** -24 * ref.abs()
    tol = tol + torch.finfo(got.dtype).eps / 2 * (ref.abs() + tol) + 1e-37
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), "%d of %d off, worst %.3g (allowed %.3g) at %s" % (
        bad.sum(), bad.numel(), (got.double() - ref).abs()[bad].max(), tol[bad].min(), bad.nonzero()[0].tolist())


def make(n, k, o, dtype, seed=0, groups=None):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + n + 3 * k + 7 * o)
    x = torch.randn(n, k, generator=g, device="cuda").to(dtype)
    shape = (o, k) if groups is None else (groups, o, k)
    W = (torch.randn(*shape, generator=g, device="cuda") * k ** -0.5).to(dtype)
    b = torch.randn(*shape[:-1], generator=g, device="cuda") * 0.1
    r = torch.randn(n, o, generator=g, device="cuda")
    return x, W, b, r


SIZES = [(1, 8, 1), (1, 256, 1024), (1, 4096, 500), (2, 72, 33), (3, 1032, 129), (4, 4544, 640), (7, 200, 4096), (8, 64, 16), (9, 520, 257),
         (13, 2056, 48), (16, 128, 1000), (17, 1096, 130), (31, 4096, 96), (32, 520, 4544), (33, 776, 100), (64, 2048, 264), (65, 136, 128),
         (100, 264, 127), (128, 512, 512), (129, 1024, 384), (255, 640, 72), (257, 264, 300), (300, 4544, 256), (513, 72, 1025),
         (777, 328, 272), (1500, 256, 2000), (2049, 1288, 520), (20, 8, 40), (200, 16, 300), (1300, 24, 4100)]


@gpu
@pytest.mark.parametrize("n,k,o", SIZES)
def test_linear_matches_definition(n, k, o):
    x, W, b, r = make(n, k, o, BF)
    for act, bias, res, out in ((NONE, None, None, F32), (TANH, b, None, BF), (ERF, b, r.to(BF), BF), (RELU, None, r, F32)):
        y = T.tardis_linear(x, W, bias=bias, act=act, residual=res, out_dtype=out)
        ref, tol = product64(x, W, bias, act, out)
        check(y, ref, tol, res)


@gpu
@pytest.mark.parametrize("n,k,o", [(1, 8, 1), (1, 256, 1024), (5, 1024, 300), (17, 40, 65), (64, 256, 1024), (130, 72, 200), (700, 512, 333), (1100, 256, 1024)])
def test_linear_fp32_matches_definition(n, k, o):
    x, W, b, r = make(n, k, o, F32)
    for act, bias, res in ((NONE, None, None), (TANH, b, r), (ERF, b, None), (RELU, None, r)):
        check(T.tardis_linear(x, W, bias=bias, act=act, residual=res), *product64(x, W, bias, act), res)


# more tiles than CTAs, pairs of CTAs, ragged ends on both sides, many channels with few outputs
@gpu
@pytest.mark.parametrize("n,k,o", [(4096, 2048, 4096), (1000, 4544, 18176), (2500, 4096, 3000), (5000, 512, 8192), (64, 16384, 4096), (200, 18176, 4544),
                                   (12, 8192, 8192), (24, 16384, 2048), (90, 16384, 264), (20000, 136, 200)])
def test_linear_large(n, k, o):
    x, W, b, r = make(n, k, o, BF)
    r = r.to(BF)
    y = T.tardis_linear(x, W, bias=b, act=TANH, residual=r)
    ref, tol = product64(x, W, b, TANH)
    check(y, ref, tol, r)


@gpu
@pytest.mark.parametrize("n,k,o", [(n, k, o) for n in (1, 8, 20, 64, 100, 200, 700) for k, o in ((11752, 96), (18176, 1000), (1904, 300))]
                         + [(1500, 1904, 4100), (2100, 8192, 2048)])
def test_fp32_outputs_of_many_channels_are_as_near_as_fp32_sums(n, k, o):
    """The tensor cores cut sums off towards zero.  A plain sum of k terms in fp32 is off by some sqrt(k) / 2 roundings of 2^-24 of it, at random; 512 channels of
    cut-off sums lose at most 32 times 2^-24 of their part, on average a third of that: 1e-6 is above both and below what k / 16 cut-offs lose (2.4e-6 of 1904 channels, 1.1e-5 of 11752)."""
    x, W, b, r = make(n, k, o, BF)
    for res in (None, r):
        y = T.tardis_linear(x, W, bias=b, residual=res, out_dtype=F32)
        ref, tol = product64(x, W, b, NONE, F32)
        check(y, ref, tol, res)
        assert (y.double() - (ref if res is None else ref + res.double())).norm() <= 1e-6 * ref.norm()
    off = offsets_of([n // 2, 0, n - n // 2])
    We = W[None].expand(3, o, k).contiguous()
    y = T.tardis_grouped_linear(x, We, off, rows=torch.arange(n, device="cuda").int(), out_dtype=F32)
    ref, tol = product64(x, W, None, NONE, F32)
    check(y, ref, tol)
    assert (y.double() - ref).norm() <= 1e-6 * ref.norm()


@gpu
@pytest.mark.parametrize("n", [1, 6, 30, 70, 500])
def test_linear_strides_in_place_and_untouched_surroundings(n):
    """Leading dimensions of their own, odd starts of y, columns behind k that hold NaN, y = residual, nothing written beside y."""
    k, o = 264, 131
    g = torch.Generator(device="cuda").manual_seed(n)
    xb = torch.full((n + 2, k + 40), float("nan"), device="cuda", dtype=BF)
    wb = torch.full((o + 2, k + 16), float("nan"), device="cuda", dtype=BF)
    x, W = xb[1:n + 1, 8:8 + k], wb[1:o + 1, :k]
    x.copy_(torch.randn(n, k, generator=g, device="cuda"))
    W.copy_(torch.randn(o, k, generator=g, device="cuda") * 0.05)
    big = torch.randn(n + 2, o + 7, generator=g, device="cuda").to(BF)
    before = big.clone()
    y = big[1:n + 1, 3:3 + o]
    res = y.clone()
    ref, tol = product64(x, W, None, ERF)
    assert T.tardis_linear(x, W, act=ERF, residual=y, out=y) is y
    check(y, ref, tol, res)
    y.copy_(before[1:n + 1, 3:3 + o])
    assert torch.equal(big, before)


@gpu
@pytest.mark.parametrize("n", [2, 20, 300])
def test_linear_special_values_stay_in_their_rows(n):
    """Infinities and NaN of one token reach that token's outputs only; those of one weight row that output only."""
    x, W, b, r = make(n, 256, 200, BF)
    x[1, 5] = float("nan")
    W[7, 3] = float("inf")
    y = T.tardis_linear(x, W, bias=b, act=RELU)
    assert y[1].isnan().all()
    keep = torch.ones(n, 200, dtype=torch.bool, device="cuda")
    keep[1] = False
    keep[:, 7] = False
    assert y[keep].isfinite().all()
    other = torch.arange(n, device="cuda") != 1
    s = x[other, 3].float()
    want = torch.where(s > 0, math.inf, torch.where(s < 0, 0.0, math.nan))
    assert torch.equal(y[other, 7].float().nan_to_num(nan=-1.0, posinf=9.0), want.nan_to_num(nan=-1.0, posinf=9.0))


@gpu
def test_linear_offsets_beyond_32_bits():
    """Rows whose first element lies beyond 2^31 elements, of y and of x."""
    k, o, ld = 64, 40, 32768
    n = 2 ** 31 // ld + 70
    big = torch.zeros(n, ld, dtype=BF, device="cuda")
    x, W, b, _ = make(n, k, o, BF)
    y = big[:, 5:5 + o]
    T.tardis_linear(x, W, bias=b, out=y)
    ref, tol = product64(x, W, b, NONE)
    check(y, ref, tol)
    big[:, 64:64 + k] = x
    T.tardis_linear(big[:, 64:64 + k], W, bias=b, out=y)
    check(y, ref, tol)


@gpu
def test_linear_runs_alike_on_streams_and_in_graphs():
    for n in (1, 12, 80, 600):
        x, W, b, r = make(n, 512, 640, BF)
        r = r.to(BF)
        want = T.tardis_linear(x, W, bias=b, act=TANH, residual=r)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        y = torch.empty_like(want)
        T.tardis_linear(x, W, bias=b, act=TANH, residual=r, out=y, stream=s)
        s.synchronize()
        assert torch.equal(y, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            T.tardis_linear(x, W, bias=b, act=TANH, residual=r, out=y)
        x.mul_(0.5)
        want2 = T.tardis_linear(x, W, bias=b, act=TANH, residual=r)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want2) and not torch.equal(want, want2)


# ---- groups -----------------------------------------------------------------------------------------------------
GROUPS = [
    [1], [0, 1], [2, 0, 0, 3], [1] * 8, [8, 8], [0, 0, 20, 0], [5, 17, 1, 33, 0, 64], [3] * 40, [100, 0, 7], [128, 129, 1, 255],
    [300, 20, 1, 0, 700, 33], [0] * 33 + [9] + [0] * 40 + [260], [2000, 3, 900],
]


def offsets_of(sizes, first=0):
    return torch.tensor(np.cumsum([first] + list(sizes)), dtype=torch.int32, device="cuda")


@gpu
@pytest.mark.parametrize("sizes", GROUPS)
@pytest.mark.parametrize("k,o", [(264, 200), (1032, 48)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_grouped_matches_definition(sizes, k, o, dtype):
    n, behind = sum(sizes), 5
    x, W, b, r = make(n + behind, k, o, dtype, groups=len(sizes))
    r = r.to(dtype)
    off = offsets_of(sizes)
    g = torch.Generator(device="cuda").manual_seed(n)
    rows = torch.randint(0, n + behind, (n + behind,), generator=g, device="cuda", dtype=torch.int32)
    x[n:] = float("nan")                                       # rows in no group, or picked by rows
    rows[rows >= n] = max(0, n - 1)
    for act, bias, res, take in ((NONE, None, None, None), (TANH, b, None, rows), (ERF, b, r, rows), (RELU, None, r, None)):
        y = torch.full((n + behind, o), 7.0, dtype=dtype, device="cuda")
        T.tardis_grouped_linear(x, W, off, bias=bias, act=act, rows=take, residual=res, out=y)
        xs = x if take is None else x[take.long()]
        at = 0
        for e, size in enumerate(sizes):
            if size:
                own = slice(at, at + size)
                check(y[own], *product64(xs[own], W[e], None if bias is None else bias[e], act), None if res is None else res[own])
            at += size
        assert (y[n:] == 7).all()


@gpu
@pytest.mark.parametrize("sizes,k,o", [([700, 1500, 0, 4000], 2048, 1024), ([300, 1800, 0, 401], 264, 4200), ([90] * 16, 1024, 2048), ([1, 0, 1, 2], 4096, 4544), ([1400, 30, 2], 4544, 520),
                                       ([9, 0, 14, 25, 3, 0, 1, 44], 4096, 1024)])
def test_grouped_large(sizes, k, o):
    test_grouped_matches_definition(sizes, k, o, BF)


@gpu
@pytest.mark.parametrize("n", [6, 40, 400])
def test_grouped_whatever_offsets_and_rows_hold(n):
    """Offsets out of order and range, row indices out of range: groups are clamped, missing rows are zeros, nothing else is written."""
    x, W, b, _ = make(n, 72, 40, BF, groups=4)
    for off, clamped in (([-5, n // 2, 1, n + 9, 2 ** 31 - 1], [0, n // 2, n // 2, n, n]), ([2, 2, n - 1, 0, 3], [2, 2, n - 1, n - 1, n - 1]),
                         ([n, 0, 0, 0, 0], [n] * 5)):
        rows = torch.arange(n, dtype=torch.int32, device="cuda")
        rows[0], rows[n // 2], rows[n - 1] = -1, n, 2 ** 31 - 1
        xs = x.clone()
        xs[[0, n // 2, n - 1]] = 0
        y = torch.full((n, 40), 7.0, dtype=BF, device="cuda")
        T.tardis_grouped_linear(x, W, torch.tensor(off, dtype=torch.int32, device="cuda"), bias=b, rows=rows, out=y)
        for e in range(4):
            lo, hi = clamped[e], clamped[e + 1]
            if hi > lo:
                check(y[lo:hi], *product64(xs[lo:hi], W[e], b[e], NONE))
        assert (y[:clamped[0]] == 7).all() and (y[clamped[4]:] == 7).all()


@gpu
@pytest.mark.parametrize("sizes_at,n", [({3: 2, 1000: 1, 1023: 3}, 6), ({0: 40, 511: 1, 512: 300, 1023: 20}, 361)])
def test_grouped_with_1024_experts(sizes_at, n):
    k, o = 64, 24
    x, W, b, _ = make(n, k, o, BF, groups=1024)
    for dtype in (BF, F32):
        xd, Wd = x.to(dtype), W.to(dtype)
        y = T.tardis_grouped_linear(xd, Wd, offsets_of([sizes_at.get(e, 0) for e in range(1024)]), bias=b)
        at = 0
        for e, size in sorted(sizes_at.items()):
            check(y[at:at + size], *product64(xd[at:at + size], Wd[e], b[e], NONE))
            at += size


@gpu
@pytest.mark.parametrize("n", [5, 40, 2000])
def test_grouped_rows_of_a_tiny_x(n):
    """Two rows of x, picked again and again."""
    x, W, b, _ = make(2, 72, 4100, BF, groups=3)
    rows = (torch.arange(n, device="cuda") % 3).int()          # 2: no such row
    xs = torch.cat([x, torch.zeros_like(x[:1])])[rows.long()]
    sizes = [n // 2, 1, n - n // 2 - 1]
    y = T.tardis_grouped_linear(x, W, offsets_of(sizes), bias=b, rows=rows)
    at = 0
    for e, size in enumerate(sizes):
        check(y[at:at + size], *product64(xs[at:at + size], W[e], b[e], NONE))
        at += size


@gpu
def test_grouped_gathers_once_whatever_offsets_hold():
    """The long form with scratch: offsets that fall again still leave the rows in front of the fall in their groups."""
    n, k, o = 2048, 72, 4104
    x, W, b, _ = make(n, k, o, BF, groups=3)
    rows = torch.randperm(n, device="cuda").int()
    rows[5], rows[1900] = -3, n
    xs = x[rows.long().clamp(0, n - 1)].clone()
    xs[5] = xs[1900] = 0
    y = torch.full((n, o), 7.0, dtype=BF, device="cuda")
    T.tardis_grouped_linear(x, W, torch.tensor([1, 1000, 2000, 30], dtype=torch.int32, device="cuda"), bias=b, rows=rows, out=y)
    check(y[1:1000], *product64(xs[1:1000], W[0], b[0], NONE))
    check(y[1000:2000], *product64(xs[1000:2000], W[1], b[1], NONE))
    assert (y[0] == 7).all() and (y[2000:] == 7).all()


@gpu
def test_combine_without_rows_and_without_tokens():
    W, r = torch.randn(2, 24, 64, device="cuda").bfloat16(), torch.randn(3, 24, device="cuda").bfloat16()
    off, slots, w = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.full((3, 2), -1, dtype=torch.int32, device="cuda"), torch.zeros(3, 2, device="cuda")
    y = T.tardis_grouped_linear_combine(W.new_empty(0, 64), W, off, slots, w, residual=r)
    assert torch.equal(y, r)
    assert T.tardis_grouped_linear_combine(W.new_empty(0, 64), W, off, slots[:0], w[:0]).shape == (0, 24)
    assert T.tardis_grouped_linear(W.new_empty(0, 64), W, off).shape == (0, 24)
    assert T.tardis_linear(W.new_empty(0, 64), W[0]).shape == (0, 24)


@gpu
def test_calls_on_another_stream_use_its_memory():
    """Results and scratch made for a call on a given stream, while the current stream is busy with memory that it has given back."""
    s = torch.cuda.Stream()
    tokens, experts, k, o = 3000, 8, 64, 4104
    logits = torch.randn(tokens, experts, device="cuda")
    x, W, b, _ = make(tokens, k, o, BF, groups=experts)
    want_route = T.tardis_route(logits, 2)
    want = T.tardis_grouped_linear(x, W, want_route[2], bias=b, rows=want_route[3])
    _, W2, _, _ = make(1, o, 72, BF, groups=experts)
    want_back = T.tardis_grouped_linear_combine(want, W2, want_route[2], want_route[4], want_route[1])
    torch.cuda.synchronize()
    a = torch.randn(4096, 4096, device="cuda")
    for _ in range(3):
        for _ in range(10):
            a @ a                                              # its result goes back to the current stream's memory at once
        route = T.tardis_route(logits, 2, stream=s)
        y = T.tardis_grouped_linear(x, W, route[2], bias=b, rows=route[3], stream=s)
        back = T.tardis_grouped_linear_combine(y, W2, route[2], route[4], route[1], stream=s)
        s.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(route, want_route)) and torch.equal(y, want) and torch.equal(back, want_back)


@gpu
def test_grouped_strided_weights_and_outputs():
    for n in (5, 50, 300):
        x, _, b, _ = make(n, 136, 65, BF, groups=3)
        Wb = torch.full((3, 70, 160), float("nan"), device="cuda", dtype=BF)
        W = Wb[:, 2:67, 8:144]
        W.copy_(torch.randn(3, 65, 136, device="cuda") * 0.1)
        yb = torch.full((n, 90), 7.0, device="cuda", dtype=BF)
        y = yb[:, 1:66]
        sizes = [n // 3, 0, n - n // 3]
        T.tardis_grouped_linear(x, W, offsets_of(sizes), bias=b, out=y)
        check(y[:n // 3], *product64(x[:n // 3], W[0], b[0], NONE))
        check(y[n // 3:], *product64(x[n // 3:], W[2], b[2], NONE))
        assert (yb[:, 0] == 7).all() and (yb[:, 66:] == 7).all()


def routed(tokens, experts, top_k, seed, masked=()):
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = torch.randn(tokens, experts, generator=g, device="cuda")
    for t in masked:
        logits[t] = -math.inf
    return logits, T.tardis_route(logits, top_k)


@gpu
@pytest.mark.parametrize("tokens,experts,top_k,k,o", [(1, 8, 2, 512, 200), (5, 4, 4, 264, 129), (30, 16, 3, 1024, 72), (300, 6, 2, 512, 300),
                                                     (1100, 9, 2, 256, 1032), (48, 64, 4, 2048, 256)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_combine_matches_definition(tokens, experts, top_k, k, o, dtype):
    _, (_, w, off, rows, slots) = routed(tokens, experts, top_k, tokens, masked=[tokens - 1] if tokens > 3 else [])
    n = tokens * top_k
    x, W, b, r = make(n, k, o, dtype, groups=experts)
    r = r[:tokens].to(dtype)
    f = torch.zeros(n, o, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(f)
    ends = off.tolist()
    act = TANH if tokens % 2 else NONE
    for e in range(experts):
        own = slice(ends[e], ends[e + 1])
        f[own], tol[own] = product64(x[own], W[e], b[e], act)
    x[ends[-1]:] = float("nan")
    for res in (None, r):
        work = torch.full((n, (o + 7) // 8 * 8), float("nan"), device="cuda")
        y = T.tardis_grouped_linear_combine(x, W, off, slots, w, bias=b, act=act, residual=res, work=work)
        there = (slots >= 0)[:, :, None]
        pick = slots.long().clamp(min=0)
        ref = torch.where(there, f[pick] * w.double()[:, :, None], 0.0)
        err = torch.where(there, tol[pick] * w.double()[:, :, None], 0.0) + top_k * 2.0 ** -23 * ref.abs()
        check(y, ref.sum(1), err.sum(1), res)


# ---- router -----------------------------------------------------------------------------------------------------
def route64(logits, top_k, normalise):
    l = logits.double().cpu().numpy()
    n, e = l.shape
    experts = np.full((n, top_k), -1, np.int64)
    weights = np.zeros((n, top_k))
    for t in range(n):
        row = [(-v, i) for i, v in enumerate(l[t]) if v > -math.inf]          # (NaN compares false)
        row.sort()
        if not row:
            continue
        top = -row[0][0]
        share = [1.0 if -v == top else math.exp(-v - top) for v, _ in row]
        total = sum(share[:top_k] if normalise else share)
        for j, (_, i) in enumerate(row[:top_k]):
            experts[t, j], weights[t, j] = i, share[j] / total
    pairs = sorted((experts[t, j], t, j) for t in range(n) for j in range(top_k) if experts[t, j] >= 0)
    rows = np.full(n * top_k, -1, np.int64)
    slots = np.full((n, top_k), -1, np.int64)
    for place, (i, t, j) in enumerate(pairs):
        rows[place], slots[t, j] = t, place
    offsets = np.searchsorted([p[0] for p in pairs], np.arange(e + 1))
    return experts, weights, offsets, rows, slots


def check_route(logits, top_k, normalise):
    got = T.tardis_route(logits, top_k, normalise=normalise)
    want = route64(logits, top_k, normalise)
    for i in (0, 2, 3, 4):
        assert np.array_equal(got[i].cpu().numpy(), want[i]), ("experts", "weights", "offsets", "rows", "slots")[i]
    # exponential (2 ulp), a sum of up to 1024 of them in a tree of at most 32 + 5 additions, a division
    w = got[1].double().cpu().numpy()
    assert (np.abs(w - want[1]) <= 45 * 2.0 ** -24 * want[1] + 1e-37).all()


@gpu
@pytest.mark.parametrize("tokens,experts,top_k", [(1, 1, 1), (1, 8, 2), (4, 8, 8), (3, 33, 4), (31, 64, 6), (127, 5, 2), (128, 256, 8), (129, 8, 2), (500, 100, 3),
                                                  (1000, 1024, 32), (2000, 40, 1)])
@pytest.mark.parametrize("normalise", [True, False])
def test_route_matches_definition(tokens, experts, top_k, normalise):
    g = torch.Generator(device="cuda").manual_seed(tokens + experts)
    big = torch.randn(tokens, experts + 3, generator=g, device="cuda") * 3
    logits = big[:, 1:1 + experts]
    check_route(logits, top_k, normalise)
    # ties, masked experts and tokens, the type's lowest value, NaN, infinities, zeros of both signs
    logits.copy_(torch.round(logits))
    logits[torch.rand(tokens, experts, generator=g, device="cuda") < 0.3] = -math.inf
    logits[torch.rand(tokens, experts, generator=g, device="cuda") < 0.1] = math.nan
    logits[torch.rand(tokens, experts, generator=g, device="cuda") < 0.1] = torch.finfo(F32).min
    logits[torch.rand(tokens, experts, generator=g, device="cuda") < 0.1] = -0.0
    logits[torch.rand(tokens, experts, generator=g, device="cuda") < 0.02] = math.inf
    logits[tokens // 2] = -math.inf
    if tokens > 2:
        logits[tokens - 1] = math.nan
    check_route(logits, top_k, normalise)


@gpu
def test_route_more_tokens_than_one_pass_of_all_blocks():
    """Above 32768 tokens a block takes several passes; checked by the definition's properties in whole-array form."""
    tokens, experts, top_k = 40001, 12, 2
    logits = torch.randn(tokens, experts, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    chosen, w, off, rows, slots = T.tardis_route(logits, top_k)
    top, idx = logits.sort(dim=1, descending=True, stable=True)
    assert torch.equal(chosen.long(), idx[:, :top_k])
    order = torch.argsort(chosen.reshape(-1).long(), stable=True)
    assert torch.equal(rows.long(), order // top_k)
    assert torch.equal(slots.reshape(-1).long()[order], torch.arange(tokens * top_k, device="cuda"))
    assert off.tolist() == [0] + torch.bincount(chosen.reshape(-1).long(), minlength=experts).cumsum(0).tolist()


@gpu
def test_route_of_no_tokens():
    chosen, w, off, rows, slots = T.tardis_route(torch.empty(0, 6, device="cuda"), 2)
    assert chosen.shape == (0, 2) and rows.numel() == 0 and off.tolist() == [0] * 7


# ---- together ---------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("tokens", [1, 3, 40, 600])
def test_block_of_experts_beside_a_dense_one(tokens):
    """A dense FFN, then a router and an FFN split over experts, on one residual stream, as one captured graph: the experts' part
    against the definition on the router's own decisions."""
    d, h, experts, top_k = 256, 512, 6, 2
    x, W1, b1, _ = make(tokens, d, h, BF, seed=1)
    _, W2, b2, _ = make(tokens, h, d, BF, seed=2)
    _, We1, be1, _ = make(1, d, h, BF, seed=3, groups=experts)
    _, We2, be2, _ = make(1, h, d, BF, seed=4, groups=experts)
    _, Wr, _, _ = make(1, d, experts, BF, seed=5)

    def block():
        u = T.tardis_linear(x, W1, bias=b1, act=TANH)
        s = T.tardis_linear(u, W2, bias=b2, residual=x)
        logits = T.tardis_linear(s, Wr, out_dtype=F32)
        _, w, off, rows, slots = T.tardis_route(logits, top_k)
        v = T.tardis_grouped_linear(s, We1, off, bias=be1, act=TANH, rows=rows)
        return u, s, logits, w, off, rows, slots, v, T.tardis_grouped_linear_combine(v, We2, off, slots, w, bias=be2, residual=s)

    block()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        u, s, logits, w, off, rows, slots, v, y = block()
    for scale in (1.0, -0.7):
        x.mul_(scale)
        graph.replay()
        torch.cuda.synchronize()
        check(u, *product64(x, W1, b1, TANH))
        check(s, *product64(u, W2, b2, NONE), x)
        check(logits, *product64(s, Wr, None, NONE))
        want = route64(logits, top_k, True)
        assert np.array_equal(rows.cpu().numpy(), want[3]) and np.array_equal(slots.cpu().numpy(), want[4])
        f = torch.zeros(tokens * top_k, d, dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(f)
        ends = off.tolist()
        for e in range(experts):
            own = slice(ends[e], ends[e + 1])
            check(v[own], *product64(s[rows.long()[own]], We1[e], be1[e], TANH))
            f[own], tol[own] = product64(v[own], We2[e], be2[e], NONE)
        pick, ww = slots.long(), w.double()[:, :, None]
        check(y, (f[pick] * ww).sum(1), (tol[pick] * ww + 2.0 ** -22 * (f[pick] * ww).abs()).sum(1), s)


# ---- refusals (no device needed) --------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def lib():
    from paper_2501_10054_b200 import build
    build.build()
    return T.load_library()


LINEAR = dict(n=4, k=64, o=24, dtype=1, out_dtype=1, act=-1, x=1 << 20, ldx=64, W=1 << 21, ldw=64, bias=None, residual=None, ldr=0, y=1 << 22, ldy=24)


@pytest.mark.parametrize("change", [
    dict(n=-1), dict(n=(1 << 31) - 4096), dict(k=0), dict(k=(1 << 30) + 8, ldx=1 << 31, ldw=1 << 31), dict(o=(1 << 30) + 1, ldy=1 << 31), dict(k=60), dict(o=0), dict(dtype=2), dict(dtype=0, out_dtype=1), dict(out_dtype=3), dict(act=3),
    dict(act=-2), dict(x=None), dict(W=None), dict(y=None), dict(x=(1 << 20) + 8), dict(W=(1 << 21) + 2), dict(ldx=56), dict(ldx=68),
    dict(ldw=60), dict(ldy=23), dict(y=(1 << 22) + 1), dict(residual=(1 << 23) + 1, ldr=24), dict(residual=1 << 23, ldr=20), dict(bias=(1 << 23) + 2),
    dict(y=(1 << 20) + 16), dict(y=1 << 21), dict(residual=(1 << 22) + 2, ldr=24), dict(residual=1 << 22, ldr=32), dict(y=1 << 22, bias=(1 << 22) + 4),
    dict(ldx=1 << 40), dict(out_dtype=0, y=(1 << 22) + 2)])
def test_linear_refuses(lib, change):
    import ctypes
    assert lib.tardis_linear(None, None) == 1
    assert lib.tardis_linear(ctypes.byref(T.LinearDesc(**{**LINEAR, **change})), None) == 1


def test_linear_of_nothing_is_fine(lib):
    import ctypes
    assert lib.tardis_linear(ctypes.byref(T.LinearDesc(**{**LINEAR, "n": 0, "x": None, "y": None})), None) == 0


GROUPED = dict(n_rows=6, n_experts=3, k=64, o=24, dtype=1, out_dtype=1, act=-1, x=1 << 20, ldx=64, n_x=6, W=1 << 21, ldw=64, stride_w=24 * 64,
               bias=None, offsets=1 << 23, rows=None, residual=None, ldr=0, y=1 << 22, ldy=24, n_tokens=0, top_k=0, slots=None, weights=None,
               work=None, work_bytes=0)
BACK = dict(n_tokens=3, top_k=2, slots=1 << 24, weights=1 << 25, work=1 << 26, work_bytes=6 * 24 * 4)


@pytest.mark.parametrize("change", [
    dict(n_rows=-1), dict(n_experts=0), dict(n_x=5), dict(n_x=-1), dict(offsets=None), dict(offsets=(1 << 23) + 2), dict(rows=(1 << 23) + 1),
    dict(stride_w=24 * 64 - 8), dict(stride_w=24 * 64 + 4), dict(k=65), dict(act=9), dict(y=1 << 20), dict(W=None), dict(slots=1 << 24), dict(weights=1 << 24),
    dict(BACK, top_k=0), dict(BACK, work=None), dict(BACK, work_bytes=6 * 24 * 4 - 1), dict(BACK, work=(1 << 26) + 4), dict(BACK, slots=(1 << 24) + 2),
    dict(BACK, weights=None), dict(BACK, n_tokens=-1)])
def test_grouped_refuses(lib, change):
    import ctypes
    assert lib.tardis_grouped_linear(None, None) == 1
    assert lib.tardis_grouped_linear(ctypes.byref(T.GroupedDesc(**{**GROUPED, **change})), None) == 1


def test_grouped_refuses_more_experts_than_it_has_room_for(lib):
    import ctypes
    assert lib.tardis_grouped_linear(ctypes.byref(T.GroupedDesc(**{**GROUPED, "n_experts": 1025})), None) == 2
    assert lib.tardis_grouped_linear(ctypes.byref(T.GroupedDesc(**{**GROUPED, "n_rows": 0})), None) == 0


def test_route_refuses(lib):
    p = [1 << 20, 1 << 21, 1 << 22, 1 << 23, 1 << 24]

    def route(n=4, e=8, k=2, norm=1, logits=1 << 19, ldl=8, outs=p, work=None, bytes=0):
        return lib.tardis_route(n, e, k, norm, logits, ldl, *outs, work, bytes, None)

    assert route(n=-1) == 1 and route(e=0) == 1 and route(k=0) == 1 and route(k=9) == 1 and route(norm=2) == 1 and route(ldl=7) == 1
    assert route(logits=None) == 1 and route(logits=(1 << 19) + 1) == 1
    for i in range(5):
        assert route(outs=p[:i] + [None] + p[i + 1:]) == 1 and route(outs=p[:i] + [p[i] + 2] + p[i + 1:]) == 1
    assert route(n=129) == 1 and route(n=129, work=1 << 25, bytes=4096 * 8 - 1) == 1
    assert route(e=1025, ldl=1025) == 2 and route(e=64, k=33, ldl=64) == 2 and route(n=1 << 30) == 2


def test_packed_descriptors_have_the_layout_of_the_structures():
    import ctypes
    assert len(T._PACK_LINEAR(*range(15))) == ctypes.sizeof(T.LinearDesc) and len(T._PACK_GROUPED(*range(26))) == ctypes.sizeof(T.GroupedDesc)
    for pack, desc in ((T._PACK_LINEAR, T.LinearDesc), (T._PACK_GROUPED, T.GroupedDesc)):
        d = desc.from_buffer_copy(pack(*range(1, len(desc._fields_) + 1)))
        assert [getattr(d, name) for name, _ in desc._fields_] == list(range(1, len(desc._fields_) + 1))


@gpu
def test_binding_refuses():
    x, W, b, r = make(4, 64, 24, BF)
    for call in (lambda: T.tardis_linear(x.cpu(), W), lambda: T.tardis_linear(x, W.float()), lambda: T.tardis_linear(x, W, bias=b.to(BF)),
                 lambda: T.tardis_linear(x, W, bias=b[:5]), lambda: T.tardis_linear(x.t(), W), lambda: T.tardis_linear(x, W, residual=r),
                 lambda: T.tardis_linear(x, W[:, :56]), lambda: T.tardis_linear(x, W, residual=r.to(BF)[:1].expand(4, 24)),
                 lambda: T.tardis_linear(x.half(), W.half()), lambda: T.tardis_linear(x[:1].expand(4, 64), W),
                 lambda: T.tardis_linear(x, W, out=torch.empty(4, 24, device="cuda"), out_dtype=BF),
                 lambda: T.tardis_grouped_linear(x, W[None], torch.zeros(2, device="cuda")),
                 lambda: T.tardis_grouped_linear(x, W[None], torch.zeros(3, device="cuda", dtype=torch.int32)),
                 lambda: T.tardis_route(x, 2), lambda: T.tardis_route(b[None], 25), lambda: T.tardis_route(b, 2)):
        with pytest.raises(T.TardisError):
            call()
