"""fdd_token_logprobs at both ends of the range of temperatures, and refusals beyond it.  The reference divides by what the library
multiplies with, 1 / temperature in fp32; tolerances as in test_gpu_logprobs.py."""
import ctypes as C

import numpy as np
import pytest
import torch

import fdd_workloads as W
from tests.gpu_util import print_case, to_dev
from tests.test_gpu_logprobs import reference
from tests.test_gpu_logprobs_lowest import LOWEST, close
from tests.test_quant_args import lib, logp  # noqa: F401

LARGEST = 2.0 ** 120
# 1.5 / t is fp32's largest number or the next below
SMALLEST = float(np.float32(1.5) / np.finfo(np.float32).max * np.float32(1 + 2.0 ** -20))


def test_range_of_temperatures(lib):  # noqa: F811
    above = float(np.nextafter(np.float32(LARGEST), np.float32(np.inf)))
    for t in (above, 2.0 ** 127, float(np.finfo(np.float32).max), 4.3e-39, 1e-40):
        assert lib.fdd_token_logprobs(C.byref(logp(temperature=t))) == 4, t
        assert "temperature" in lib.fdd_last_error().decode()


@pytest.mark.gpu
@pytest.mark.parametrize("t", [LARGEST, 1e36, 1e30, 1e10, 1e-10, 1e-30, SMALLEST])
@pytest.mark.parametrize("dtype", [W.BF16, W.F32])
@pytest.mark.parametrize("V", [9, 700, 40007])
def test_far_temperatures(V, dtype, t):
    import paper_2605_23163_amd as F
    print_case(test="logprobs_temperature", V=V, dtype=dtype, t=t)
    rng = np.random.default_rng([V, 43])
    low = LOWEST[dtype]
    inv = float(np.float32(1) / np.float32(t))
    spread = min(t, -low / 64)           # differences that the temperature turns into ones that count
    rows = [rng.standard_normal(V) * spread, rng.standard_normal(V), np.where(rng.random(V) < 0.5, low, -low), np.where(rng.random(V) < 0.7, low, 1.0),
            np.where(rng.random(V) < 0.5, -np.inf, rng.standard_normal(V) * spread), rng.standard_normal(V) * spread + low / 2]
    for r in rows:
        r[V // 2] = max(r[V // 2], 0.0)
    x = W.to_storage(np.array([rows]), dtype)
    wide = W.widen(x, dtype).astype(np.float64)[0]
    tokens = wide.argmax(1).astype(np.int32)
    top = min(V, 6)
    lp, ent, ids, tlp = (g.cpu().numpy()[0] for g in F.fdd_token_logprobs(to_dev(x), torch.from_numpy(tokens[None]).cuda(), top=top, temperature=t))
    rlp, rent, rids, rtlp, lse = reference(wide, tokens, top, 1 / inv)
    close(lp.astype(np.float64), rlp, lse, V)
    np.testing.assert_array_equal(ids, rids)
    close(tlp.astype(np.float64), rtlp, lse[:, None], V)
    r = (V / 256 + 64) * 2.0 ** -24
    assert (np.abs(ent - rent) <= (2 * r + 2.0 ** -22) * rent + 1e-37).all()
