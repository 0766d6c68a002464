"""Attention over the 8-bit cache where values are far apart, very small, or missing.

Scores are all 0 in the first two tests, so that every probability is 1 and an output is the mean of n values, which fp32 sums to n 2^-24 of
the largest partial sum's mean.  A piece's average is kept in 16 bits: off by 2^-11 of itself, by 2^-39 of the row's largest one (the step
of fp16 below its normal numbers is 2^-24, half of that is the error, and the largest one lies at 2^14 or above), or by 2^-126 (rows below
2^-87 are scaled by 2^101, half a step is 2^-25).  The output is rounded to bf16, 2^-8 of itself."""
import numpy as np
import pytest
import torch

import fdd_workloads as W
from tests.gpu_util import print_case, rand_attn, to_dev, to_f64
from tests.test_gpu_quant import F, cached  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("splits", [1, 2, 7])
@pytest.mark.parametrize("D,N,low", [(64, 1, -20), (128, 1, -36), (128, 12, -36), (64, 3, -60)])
def test_channels_far_apart(F, D, N, low, splits):  # noqa: F811
    """Extension and block carry channels of 2^0 down to 2^low beside one another; the cache's values have a scale for 64 rows, so that its small ones
    are 0 or coarse codes: the reference takes the values as the cache holds them."""
    print_case(test="quant_attn_channels", D=D, N=N, low=low, splits=splits)
    rng = np.random.default_rng([D, N, -low])
    B, L, Hq, Hkv = 8, 640, 8, 2
    d = rand_attn(rng, N, B, L, Hq, Hkv, D, W.BF16)
    spread = np.exp2(np.rint(np.linspace(0, low, D)))[rng.permutation(D)]
    d["prefix_v"] = W.to_storage(rng.uniform(1.0, 2.0, (L, Hkv, D)) * spread, W.BF16)
    d["block_v"] = W.to_storage(rng.uniform(1.0, 2.0, (N, B, Hkv, D)) * spread, W.BF16)
    compare(F, d, L, B, Hq, Hkv, splits)


@pytest.mark.parametrize("splits", [1, 2, 7])
@pytest.mark.parametrize("exponent", [-112, -105, -88, 100])
def test_small_and_large_rows(F, exponent, splits):  # noqa: F811
    print_case(test="quant_attn_small", exponent=exponent, splits=splits)
    rng = np.random.default_rng(exponent + 200)
    N, B, L, Hq, Hkv, D = 2, 8, 640, 8, 2, 128
    d = rand_attn(rng, N, B, L, Hq, Hkv, D, W.BF16)
    d["prefix_v"] = W.to_storage(np.ldexp(rng.uniform(-2.0, 2.0, (L, Hkv, D)), exponent), W.BF16)
    d["block_v"] = W.to_storage(np.ldexp(rng.uniform(-2.0, 2.0, (N, B, Hkv, D)), exponent), W.BF16)
    compare(F, d, L, B, Hq, Hkv, splits)


def compare(F, d, L, B, Hq, Hkv, splits):  # noqa: F811
    p, d = cached(F, d, W.BF16)
    dev = {k: to_dev(x) for k, x in d.items()}
    out = to_f64(F.fdd_block_attn_quant(torch.zeros_like(dev["q"]), p, L, dev["block_k"], dev["block_v"], splits=splits))
    pv, bv = (W.widen(d[k], W.BF16).astype(np.float64) for k in ("prefix_v", "block_v"))
    ref = np.repeat((pv.sum(0) + bv.sum(1, keepdims=True)) / (L + B), Hq // Hkv, axis=2)
    # the largest magnitude of each channel, and of the row
    most = np.repeat(np.maximum(np.abs(pv).max(0), np.abs(bv).max(1, keepdims=True)), Hq // Hkv, axis=2)
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + (L + B) * 2.0 ** -24) * most + 2.0 ** -39 * most.max(-1, keepdims=True) + 2.0 ** -126
    assert (np.abs(out - ref) <= tol).all(), float((np.abs(out - ref) / tol).max())


@pytest.mark.parametrize("L,row", [(200, 3), (2500, 2499)])
def test_missing_values_in_fp32(F, L, row):  # noqa: F811
    """A NaN among the values of a head reaches that channel of every row of the head; one among the keys all channels.  (bf16 leaves rows
    that see one undefined.)"""
    print_case(test="quant_attn_nan", L=L, row=row)
    d = {k: to_dev(v) for k, v in rand_attn(np.random.default_rng(L), 2, 8, L, 4, 2, 64, W.F32).items()}
    for name in ("prefix_v", "prefix_k"):
        d[name][row, 1, 5] = float("nan")
        p = F.fdd_quant_prefix(L, 2, 64)
        F.fdd_prefix_quantize(d["prefix_k"], d["prefix_v"], p)
        nan = torch.isnan(F.fdd_block_attn_quant(d["q"], p, L, d["block_k"], d["block_v"]))
        assert not bool(nan[:, :, :2].any()) and bool(nan[:, :, 2:, 5].all())
        assert bool(nan[:, :, 2:].all()) == (name == "prefix_k")
        d[name][row, 1, 5] = 0.0
