"""Attention over a paged cache in fp32: a NaN or an infinity is passed on to the rows that see it."""
import numpy as np
import pytest
import torch

from tests.test_gpu_paged_attn import Call

pytestmark = pytest.mark.gpu

# lens, mode: one piece; pieces joined by a wavefront (fewer than 24 of an M-tile) and by four of them
CALLS = [([20], "full"), ([900, 300, 2000, 700], "causal"), ([9000], "causal"), ([0, 40], "tree")]


def finite_rows(x, out):
    """Whether every row (request, token, head) of the output has finite numbers only; all others have nothing but NaN."""
    o = out.cpu().numpy()
    bad = np.isnan(o)
    assert np.all(bad.any(-1) == bad.all(-1)) and np.isfinite(o[~bad]).all()
    return ~bad.any(-1)


@pytest.mark.parametrize("case", range(len(CALLS)))
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_query(case, bad):
    lens, mode = CALLS[case]
    x = Call("f32", lens, 4, 8, 2, 64, 16, None, mode, seed=case)
    n = len(lens) - 1
    x.q[n, 2, 5, 3] = bad
    got = x.run()
    ok = finite_rows(x, got)
    assert not ok[n, 2, 5] and ok.sum() == ok.size - 1
    x.q[n, 2, 5, 3] = 0.0
    got[n, 2, 5] = x.run()[n, 2, 5]
    x.check(got)


@pytest.mark.parametrize("case", range(len(CALLS)))
def test_key_in_the_cache(case):
    lens, mode = CALLS[case]
    n = len(lens) - 1
    x = Call("f32", lens, 4, 8, 2, 64, 16, None, mode, seed=case)
    want = x.run().clone()
    at = lens[n] // 2
    x.cache.k[x.cache.page_table[n, at // 16].long(), 1, at % 16, 7] = float("nan")
    got = x.run()
    ok = finite_rows(x, got)
    assert not ok[n, :, 4:].any() and ok[n, :, :4].all() and ok[:n].all()
    assert torch.equal(got[:n], want[:n]) and torch.equal(got[n, :, :4], want[n, :, :4])


@pytest.mark.parametrize("case", range(len(CALLS)))
def test_key_of_a_token(case):
    """Rows that see the token are NaN, the others as they were (to rounding: a row's reference follows the rows next to it)."""
    lens, mode = CALLS[case]
    n = len(lens) - 1
    x = Call("f32", lens, 4, 8, 2, 64, 16, None, mode, seed=case)
    x.run()
    x.k[n, 2, 0, 0] = float("nan")
    got = x.run()
    ok = finite_rows(x, got)
    sees = x.see[n][:, 2]
    assert np.array_equal(ok[n, :, :4], np.repeat(~sees[:, None], 4, 1)) and ok[n, :, 4:].all() and ok[:n].all()
    x.k[n, 2, 0, 0] = 0.0
    clean = x.run()
    gone = torch.from_numpy(~ok).cuda()
    got[gone] = clean[gone]
    x.check(got)


def test_everything():
    x = Call("f32", [3000, 5], 4, 8, 2, 128, 64, None, "causal", seed=3)
    x.q.fill_(float("nan"))
    assert bool(torch.isnan(x.run()).all())


def test_rows_that_see_nothing_stay_zero():
    """Also beside rows that are NaN."""
    x = Call("f32", [0, 0], 9, 4, 2, 64, 16, None, "any", seed=4)
    x.q[0, 1] = float("nan")
    got = x.run()
    assert bool((got[:, ::3] == 0).all()) and bool(torch.isnan(got[0, 1]).all())
