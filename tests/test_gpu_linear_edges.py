"""The dense and expert-grouped products where their contract ends: very many channels, tails and special values of the activations, offsets that fall,
more experts than rows, rows in no group, fp32 outputs of every form.  Bounds: see the head of test_gpu_linear.py."""
import math

import numpy as np
import pytest
import torch

import paper_2501_10054_b200 as T
from tests.test_gpu_linear import BF, ERF, F32, NONE, RELU, TANH, act64, check, check_route, gpu, make, offsets_of, product64, routed


# ---- very many channels -----------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("grouped", [False, True])
def test_sums_of_very_many_channels_are_held_in_fp32(grouped):
    """2^28 and 2^24 - 1 ones: a sum to which 16 ones are added at a time and that is cut off to 24 bits (steps of 32) never takes one in, and any quarter of the channels
    is 2^-6 of the result.  512 ones at a time are whole steps: what is lost is the 511 ones beside the 2^28, 2^-19 of the result, and 2^28 + 2^24 has five bits."""
    n, k, o = 65, 2 ** 24, 8
    x = torch.ones(1 if grouped else n, k, dtype=BF, device="cuda")
    W = torch.ones(o, k, dtype=BF, device="cuda")
    x[:, 0] = W[:, 0] = 2.0 ** 14
    if grouped:
        rows, off = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
        y = T.tardis_grouped_linear(x, W[None], off, rows=rows)
        back = T.tardis_grouped_linear_combine(x, W[None], off, torch.arange(n, dtype=torch.int32, device="cuda")[:, None], torch.ones(n, 1, device="cuda"), rows=rows)
        assert (back.float() == 2.0 ** 28 + 2.0 ** 24).all()
    else:
        y = T.tardis_linear(x, W)
    assert (y.float() == 2.0 ** 28 + 2.0 ** 24).all(), y.float().unique().tolist()


@gpu
@pytest.mark.parametrize("n,k,o", [(70, 2 ** 17 + 8, 40), (100, 2 ** 17 + 200, 300), (600, 2 ** 17 + 72, 520), (300, 2 ** 17 + 8, 1032)])
def test_16_bit_outputs_of_very_many_channels(n, k, o):
    """Above 2^17 channels, in every shape of tile, with all of the epilogue."""
    x, W, b, r = make(n, k, o, BF)
    r = r.to(BF)
    for act, bias, res in ((NONE, None, None), (TANH, b, r), (ERF, b, None), (RELU, None, r)):
        ref, tol = product64(x, W, bias, act, F32)             # (the bound of fp32 sums)
        check(T.tardis_linear(x, W, bias=bias, act=act, residual=res), ref, tol, res)
    big = torch.full((n, o + 5), 7.0, dtype=BF, device="cuda")
    ref, tol = product64(x, W, b, NONE, F32)
    check(T.tardis_linear(x, W, bias=b, out=big[:, 3:3 + o]), ref, tol)
    assert (big[:, :3] == 7).all() and (big[:, 3 + o:] == 7).all()


# ---- activations ------------------------------------------------------------------------------------------------
def act_rows(z, n, dtype):
    """x [n, 8] and W [len(z), 8] whose product is z in every row, exactly (z of `dtype`)."""
    x = torch.zeros(n, 8, dtype=dtype, device="cuda")
    W = torch.zeros(len(z), 8, dtype=dtype, device="cuda")
    x[:, 0] = 1
    W[:, 0] = z
    return x, W


@gpu
@pytest.mark.parametrize("n,dtype,out", [(n, BF, out) for n in (1, 8, 40, 100, 600) for out in (BF, F32)] + [(n, F32, F32) for n in (1, 8, 40, 600)])
@pytest.mark.parametrize("act", [TANH, ERF])
def test_tails_of_the_activations(n, dtype, out, act):
    """Where 1 + tanh or 1 + erf cancels.  Relative to the value: the arguments (z^2 / 2 and about z^2 for the two forms, up to 60 of them here) round three times by 2^-24, the exponential by
    two units and one more for every 0.86 of its argument (60 / 0.86 + 2 units of 2^-23), a division and products 2^-22: 60 * 3 * 2^-24 + 72 * 2^-23 + 2^-22 < 2e-5; then the output's rounding."""
    z = -torch.arange(0.0625, 10.0, 0.0625, device="cuda").to(dtype)
    z = torch.cat([z, -z])
    x, W = act_rows(z, n, dtype)
    y = T.tardis_linear(x, W, act=act, out_dtype=out).double()
    ref = act64(z.double(), act)
    assert ((y - ref).abs() <= (2e-5 + torch.finfo(out).eps / 2 * 1.001) * ref.abs() + 1e-37).all(), (((y - ref) / ref).abs().max(dim=0).values / 2e-5).max()


@gpu
@pytest.mark.parametrize("act", [NONE, TANH, ERF, RELU])
@pytest.mark.parametrize("n,dtype", [(1, BF), (8, BF), (40, BF), (100, BF), (600, BF), (1, F32), (8, F32), (40, F32), (600, F32)])
def test_activations_of_special_values(n, dtype, act):
    """Very large values of both signs, zeros, infinities and NaN: what the definition gives (the product of -inf and 0 is NaN for the GELU forms, as in the definition)."""
    z = torch.tensor([0.0, 1e-30, -1e-30, 30.0, -30.0, 1e10, -1e10, 1e19, -1e19, 3e38, -3e38, math.inf, -math.inf, math.nan], device="cuda").to(dtype)
    x, W = act_rows(z, n, dtype)
    W[:, 1:] = 0
    for out in {dtype, F32}:
        y = T.tardis_linear(x, W, act=act, out_dtype=out).double()
        ref = act64(z.double(), act).to(out).double().expand(n, -1)
        assert torch.equal(y.isnan(), ref.isnan()) and torch.equal(y.isinf(), ref.isinf())
        fine = ref.isfinite()
        assert ((y - ref)[fine].abs() <= 2.0 ** -20 * ref[fine].abs() + (torch.finfo(out).eps * ref[fine].abs() if out == BF else 0) + 1e-37).all()


@gpu
@pytest.mark.parametrize("n,k,o", [(5, 264, 130), (20, 136, 40), (64, 2048, 264), (100, 1032, 300), (300, 264, 1000), (700, 520, 1032), (1500, 264, 2000)])
def test_fp32_outputs_of_the_gelu_forms(n, k, o):
    x, W, b, r = make(n, k, o, BF)
    for act in (TANH, ERF):
        for res in (None, r):
            check(T.tardis_linear(x, W, bias=b, act=act, residual=res, out_dtype=F32), *product64(x, W, b, act, F32), res)


# ---- second products of hundreds of rows ------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("n,k,o", [(100, 16384, 2048), (160, 16384, 4096), (256, 16384, 4096), (384, 16384, 4096), (512, 18176, 4544), (500, 11752, 1000)])
def test_second_products_of_hundreds_of_rows(n, k, o):
    x, W, b, r = make(n, k, o, BF)
    for out in (BF, F32):
        res = r.to(out)
        check(T.tardis_linear(x, W, bias=b, residual=res, out_dtype=out), *product64(x, W, b, NONE, out), res)


# ---- groups -----------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [7, 60, 700])
def test_return_with_offsets_that_fall(n, dtype):
    """Groups end where the largest offset so far is: rows that have been computed come back, whatever the last entry says."""
    x, W, b, _ = make(n, 72, 44, dtype, groups=4)
    hi = n - 2
    for off, clamped in (([1, n // 2, hi, hi, 3], [1, n // 2, hi, hi, hi]), ([1, hi, 2, n // 2, 0], [1, hi, hi, hi, hi]), ([-4, n // 2, n + 7, -1, 0], [0, n // 2, n, n, n])):
        slots = torch.arange(-2, n + 2, dtype=torch.int32, device="cuda")[:, None]
        w = torch.full((n + 4, 1), 0.5, device="cuda")
        f = torch.zeros(n + 4, 44, dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(f)
        for e in range(4):
            lo, end = clamped[e], clamped[e + 1]
            f[2 + lo:2 + end], tol[2 + lo:2 + end] = product64(x[lo:end], W[e], b[e], NONE)
        work = torch.full((n, 48), float("nan"), device="cuda")
        y = T.tardis_grouped_linear_combine(x, W, torch.tensor(off, dtype=torch.int32, device="cuda"), slots, w, bias=b, work=work)
        check(y, 0.5 * f, 0.5 * tol)


@gpu
@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("take", [False, True])
@pytest.mark.parametrize("tokens,experts,top_k,k,o", [(6, 8, 2, 264, 129), (70, 5, 3, 520, 200), (900, 6, 2, 264, 520), (1300, 4, 2, 136, 1032)])
def test_return_of_every_form(tokens, experts, top_k, k, o, take, dtype, out):
    """Both types of result, rows in their order or picked by an index."""
    _, (_, w, off, _, slots) = routed(tokens, experts, top_k, tokens)
    n = tokens * top_k
    x, W, b, r = make(n, k, o, dtype, groups=experts)
    rows = torch.randint(0, n, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n), dtype=torch.int32) if take else None
    xs = x[rows.long()] if take else x
    f = torch.zeros(n, o, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(f)
    ends = off.tolist()
    for e in range(experts):
        own = slice(ends[e], ends[e + 1])
        f[own], tol[own] = product64(xs[own], W[e], b[e], ERF, out)
    res = r[:tokens].to(out)
    y = T.tardis_grouped_linear_combine(x, W, off, slots, w, bias=b, act=ERF, rows=rows, residual=res, out_dtype=out)
    pick, ww = slots.long(), w.double()[:, :, None]
    check(y, (f[pick] * ww).sum(1), (tol[pick] * ww + top_k * 2.0 ** -23 * (f[pick] * ww).abs()).sum(1), res)


@gpu
@pytest.mark.parametrize("n,experts,o", [(12, 64, 1024), (40, 256, 300), (9, 1024, 512)])
def test_experts_without_rows_choose_no_other_kernel(n, experts, o):
    """fp32 rows of a few of many experts are computed as those of the few alone are: the same bits, whatever the number of the others."""
    k, few = 264, 8
    x, W, b, _ = make(n, k, o, F32, groups=few)
    where = torch.linspace(0, experts - 1, few, device="cuda").long()
    W_all = torch.zeros(experts, o, k, device="cuda")
    b_all = torch.zeros(experts, o, device="cuda")
    W_all[where], b_all[where] = W, b
    sizes = [n // few + (1 if i < n % few else 0) for i in range(few)]
    all_sizes = [0] * experts
    for i, e in enumerate(where.tolist()):
        all_sizes[e] = sizes[i]
    # (as many groups as rows at most are counted: the few with empty ones up to there)
    some = min(n, experts)
    W_some, b_some = torch.zeros(some, o, k, device="cuda"), torch.zeros(some, o, device="cuda")
    W_some[:few], b_some[:few] = W, b
    want = T.tardis_grouped_linear(x, W_some, offsets_of(sizes + [0] * (some - few)), bias=b_some)
    got = T.tardis_grouped_linear(x, W_all, offsets_of(all_sizes), bias=b_all)
    assert torch.equal(got, want)


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,o", [(1, 40), (3, 40), (7, 40), (20, 40), (100, 520), (1500, 4104)])
def test_rows_outside_x_are_rows_of_zeros(n, o, dtype):
    """Times infinite weights they are NaN, as zeros of x are, whichever kernel serves the call; times finite ones the bias."""
    k = 72
    x, W, b, _ = make(n, k, o, dtype, groups=1)
    W[0, 5, 3] = math.inf
    rows = torch.arange(n, dtype=torch.int32, device="cuda")
    rows[n // 2] = -1
    for out in {dtype, F32}:
        y = T.tardis_grouped_linear(x, W, torch.tensor([0, n], dtype=torch.int32, device="cuda"), bias=b, rows=rows, out_dtype=out)[n // 2]
        assert y[5].isnan()
        y[5] = b[0, 5]
        assert torch.equal(y, b[0].to(out))


@gpu
def test_group_sizes_change_between_replays():
    """One captured call; the sizes of the groups, the rows and the slots change on the device: even, all in one group, skewed, none."""
    tokens, experts, top_k, k, o = 700, 6, 2, 136, 4104
    n = tokens * top_k
    x, W, b, _ = make(tokens, k, o, BF, groups=experts)
    _, W2, b2, _ = make(1, o, 72, BF, groups=experts)
    off, rows = torch.zeros(experts + 1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    slots, w = torch.zeros(tokens, top_k, dtype=torch.int32, device="cuda"), torch.zeros(tokens, top_k, device="cuda")
    y = torch.zeros(n, o, dtype=BF, device="cuda")

    def block():
        T.tardis_grouped_linear(x, W, off, bias=b, act=RELU, rows=rows, out=y)
        return T.tardis_grouped_linear_combine(y, W2, off, slots, w, bias=b2)

    block()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        back = block()
    g = torch.Generator(device="cuda").manual_seed(3)
    for tilt in (0.0, 20.0, 3.0, -math.inf):
        logits = torch.randn(tokens, experts, generator=g, device="cuda")
        logits = torch.full_like(logits, tilt) if tilt < 0 else logits + tilt * torch.arange(experts, device="cuda") / experts
        _, w_new, off_new, rows_new, slots_new = T.tardis_route(logits, top_k)
        for dst, src in ((w, w_new), (off, off_new), (rows, rows_new), (slots, slots_new)):
            dst.copy_(src)
        y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        ends = off.tolist()
        f, tol = torch.zeros(n, 72, dtype=torch.float64, device="cuda"), torch.zeros(n, 72, dtype=torch.float64, device="cuda")
        for e in range(experts):
            own = slice(ends[e], ends[e + 1])
            if ends[e + 1] > ends[e]:
                check(y[own], *product64(x[rows.long()[own]], W[e], b[e], RELU))
                f[own], tol[own] = product64(y[own], W2[e], b2[e], NONE)
        assert (y[ends[-1]:] == 7).all()
        there, pick = (slots >= 0)[:, :, None], slots.long().clamp(min=0)
        part = torch.where(there, f[pick] * w.double()[:, :, None], 0.0)
        check(back, part.sum(1), (torch.where(there, tol[pick] * w.double()[:, :, None], 0.0) + 2.0 ** -22 * part.abs()).sum(1))


@gpu
@pytest.mark.parametrize("n", [1, 4, 8, 20, 200])
def test_weights_and_rows_written_by_the_launch_before(n):
    """A launch begins while the one before is still running: weights, rows and slots that that one writes, at the same place every time, are read as written."""
    k, o, rounds = 1024, 512, 12
    x, _, b, _ = make(n, k, o, BF)
    low = [make(o, 64, k, BF, seed=i)[0] for i in range(rounds)]
    _, up, _, _ = make(1, 64, k, BF, seed=77)                  # W = low up^T: [o, k]
    logits = [torch.randn(n, 4, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)) for i in range(rounds)]
    W, y, back = torch.zeros(4, o, k, dtype=BF, device="cuda"), torch.zeros(2 * n, o, dtype=BF, device="cuda"), torch.zeros(n, k, dtype=BF, device="cuda")
    _, W2, _, _ = make(1, o, k, BF, seed=5, groups=4)
    work = torch.zeros(2 * n, k, device="cuda")

    def step(i):
        _, w, off, rows, slots = T.tardis_route(logits[i], 2)
        for e in range(4):
            T.tardis_linear(low[i].roll(e, 0), up, out=W[e])
        T.tardis_linear(x, W[3], out=y[:n])
        first = y[:n].clone()
        T.tardis_grouped_linear(x, W, off, rows=rows, act=RELU, out=y)
        T.tardis_grouped_linear_combine(y, W2, off, slots, w, out=back, work=work)
        return first, y.clone(), back.clone()

    apart = []
    for i in range(rounds):
        got = step(i)
        torch.cuda.synchronize()
        apart.append(got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        together = [step(i) for i in range(rounds)]
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for i in range(rounds) for p, q in zip(apart[i], together[i]))


# ---- router -----------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("tokens,experts,top_k", [(1, 1024, 32), (100, 1024, 32), (128, 600, 7), (77, 300, 20), (128, 129, 1), (90, 128, 16), (200, 128, 16), (300, 64, 9), (130, 600, 32)])
@pytest.mark.parametrize("normalise", [True, False])
def test_route_of_many_experts(tokens, experts, top_k, normalise):
    g = torch.Generator(device="cuda").manual_seed(tokens + experts)
    logits = torch.randn(tokens, experts, generator=g, device="cuda") * 4
    check_route(logits, top_k, normalise)
    logits = torch.round(logits)
    logits[torch.rand(tokens, experts, generator=g, device="cuda") < 0.9] = -math.inf
    check_route(logits, top_k, normalise)


@gpu
@pytest.mark.parametrize("tokens,experts,top_k", [(65537, 64, 4), (70001, 8, 2), (150001, 5, 1), (300007, 100, 3), (40000, 200, 8)])
def test_route_of_very_many_tokens(tokens, experts, top_k):
    """Parts of 64, 128, 256 and more tokens; checked in whole-array form, with masked tokens."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    logits = torch.randn(tokens, experts, generator=g, device="cuda")
    logits[tokens - tokens // 9:] = -math.inf
    logits[1000] = -math.inf
    chosen, w, off, rows, slots = T.tardis_route(logits, top_k)
    top, idx = logits.sort(dim=1, descending=True, stable=True)
    there = top[:, :top_k] > -math.inf
    want = torch.where(there, idx[:, :top_k], experts)
    assert torch.equal(torch.where(chosen >= 0, chosen, experts).long(), want)
    order = torch.argsort(want.reshape(-1), stable=True)
    pairs = int(there.sum())
    assert torch.equal(rows.long()[:pairs], order[:pairs] // top_k) and (rows[pairs:] == -1).all()
    assert torch.equal(slots.reshape(-1).long()[order[:pairs]], torch.arange(pairs, device="cuda")) and (slots[~there] == -1).all()
    assert off.tolist() == [0] + torch.bincount(want.reshape(-1), minlength=experts)[:experts].cumsum(0).tolist()
    share = torch.where(there, torch.exp((top[:, :top_k] - top[:, :1]).double()), 0.0)
    ref = torch.where(there, share / share.sum(1, keepdim=True), 0.0)
    assert ((w.double() - ref).abs() <= 45 * 2.0 ** -24 * ref + 1e-37).all()


# ---- the binding ------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_in_no_group_of_a_fresh_output_are_zero(dtype):
    n, k, o = 300, 64, 48
    x, W, b, r = make(n, k, o, dtype, groups=2)
    for _ in range(3):
        stale = torch.full((n, o), float("nan"), dtype=dtype, device="cuda")
        del stale                                              # (the memory that a fresh output of this size gets)
        y = T.tardis_grouped_linear(x, W, torch.tensor([4, 100, 250], dtype=torch.int32, device="cuda"), bias=b)
        assert (y[:4] == 0).all() and (y[250:] == 0).all() and y.isfinite().all()
        check(y[4:100], *product64(x[4:100], W[0], b[0], NONE))


@gpu
@pytest.mark.parametrize("n,k,o,out", [(2048, 4096, 4096, F32), (1024, 2 ** 17 + 8, 4096, BF)])
def test_no_scratch_for_calls_that_use_none(n, k, o, out):
    """fp32 outputs, and 16-bit ones of very many channels, pick their rows tile by tile: n k bf16 of scratch would never be touched."""
    x, W, _, _ = make(n, k, o, BF, groups=1)
    rows, off = torch.arange(n, dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    y = torch.empty(n, o, dtype=out, device="cuda")
    T.tardis_grouped_linear(x, W, off, rows=rows, out=y)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    T.tardis_grouped_linear(x, W, off, rows=rows, out=y)
    assert torch.cuda.max_memory_allocated() == before
    check(y, *product64(x, W[0], None, NONE, F32))


@gpu
def test_binding_refuses_what_is_no_matrix_or_number():
    x, W, b, r = make(4, 64, 24, BF)
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    slots, w = torch.zeros(4, 1, dtype=torch.int32, device="cuda"), torch.zeros(4, 1, device="cuda")
    flat = torch.zeros(96, dtype=BF, device="cuda")
    for call in (lambda: T.tardis_linear(x, W, out=flat), lambda: T.tardis_linear(x, W, residual=flat), lambda: T.tardis_linear(x, W, out=flat.view(1, 4, 24)),
                 lambda: T.tardis_linear(x, W, act=None), lambda: T.tardis_linear(x, W, act=1.5), lambda: T.tardis_linear(x, W, act=1 << 40),
                 lambda: T.tardis_grouped_linear(x, W[None], off, out=flat), lambda: T.tardis_grouped_linear(x, W[None], off, residual=flat),
                 lambda: T.tardis_grouped_linear(x, W[None], off, act="relu"),
                 lambda: T.tardis_grouped_linear_combine(x, W[None], off, slots, w, residual=flat),
                 lambda: T.tardis_grouped_linear_combine(x, W[None], off, slots, w, work=torch.zeros(8, device="cuda")),
                 lambda: T.tardis_route(torch.zeros(4, 8, device="cuda"), 1.5), lambda: T.tardis_route(torch.zeros(4, 8, device="cuda"), None)):
        with pytest.raises(T.TardisError):
            call()
    assert torch.equal(T.tardis_linear(x, W, act=np.int64(RELU)), T.tardis_linear(x, W, act=RELU))          # (whole numbers of any type)
    assert T.tardis_route(torch.zeros(4, 8, device="cuda"), np.int64(3))[0].shape == (4, 3)


# ---- refusals (no device needed) --------------------------------------------------------------------------------
@pytest.mark.parametrize("change", [
    dict(work=(1 << 22) + 16), dict(work=1 << 20), dict(work=(1 << 21) + 3 * 24 * 64 * 2 - 16), dict(work=(1 << 23) - 16), dict(work=(1 << 24) - 560), dict(work=1 << 25),
    dict(residual=(1 << 26) + 64, ldr=24), dict(bias=(1 << 26) + 64), dict(rows=(1 << 26) + 572), dict(slots=(1 << 22) + 4), dict(weights=(1 << 22) + 3 * 48 - 4),
    dict(offsets=(1 << 22) + 8), dict(rows=(1 << 22) - 20)])
def test_scratch_and_indices_that_share_memory_are_refused(change):
    import ctypes

    from paper_2501_10054_b200 import build
    from tests.test_gpu_linear import BACK, GROUPED
    build.build()
    assert T.load_library().tardis_grouped_linear(ctypes.byref(T.GroupedDesc(**{**GROUPED, **BACK, **change})), None) == 1


@pytest.mark.parametrize("change", [dict(offsets=(1 << 22) + 8), dict(rows=(1 << 22) - 20), dict(rows=(1 << 22) + 284),
                                    dict(rows=1 << 24, work=(1 << 24) - 752, work_bytes=768), dict(rows=1 << 24, work=1 << 20, work_bytes=768),
                                    dict(rows=1 << 24, work=(1 << 22) + 272, work_bytes=768)])
def test_indices_and_gathered_rows_that_share_memory_are_refused(change):
    import ctypes

    from paper_2501_10054_b200 import build
    from tests.test_gpu_linear import GROUPED
    build.build()
    assert T.load_library().tardis_grouped_linear(ctypes.byref(T.GroupedDesc(**{**GROUPED, **change})), None) == 1


@gpu
def test_matrices_side_by_side_in_one_buffer_are_no_overlap():
    """Columns of one buffer that do not meet: x, residual and y, and indices between two rows of y."""
    n, k, o = 12, 64, 24
    buf = torch.randn(n, 256, device="cuda").to(BF)
    x, r, y = buf[:, :k], buf[:, k:k + o], buf[:, 96:96 + o]
    off, rows = buf[2, 128:132].view(torch.int32), buf[3, 128:152].view(torch.int32)
    off.copy_(torch.tensor([0, n], dtype=torch.int32))
    rows.copy_(torch.arange(n - 1, -1, -1, dtype=torch.int32))
    W = (torch.randn(1, o, k, device="cuda") * 0.1).to(BF)
    ref, tol = product64(x.flip(0), W[0], None, NONE)
    T.tardis_grouped_linear(x, W, off, rows=rows, residual=r, out=y)
    check(y, ref, tol, r)
    assert torch.equal(rows, torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda"))
