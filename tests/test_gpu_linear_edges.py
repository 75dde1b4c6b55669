"""The dense and expert-grouped products where their contract ends: very many channels, tails and special values of the activations, offsets that fall,
more experts than rows, rows in no group, fp32 outputs of every form.  Bounds: see the head of test_gpu_linear.py."""
import math

import numpy as np
import pytest
import torch

import paper_2501_10054_b200 as T
from tests.test_gpu_linear import BF, ERF, F32, NONE, RELU, TANH, act64, check, gpu, make, offsets_of, product64, routed


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
