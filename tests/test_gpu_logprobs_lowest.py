"""fdd_token_logprobs on rows whose entries are ruled out with the lowest finite number of their type, or are as large as it.

Tolerances as in test_gpu_logprobs.py.  A log probability below fp32's lowest number is -inf: the reference is rounded to fp32 before it
is compared, which the tolerance counts already."""
import numpy as np
import pytest
import torch

import fdd_workloads as W
from tests.gpu_util import print_case, to_dev
from tests.test_gpu_logprobs import reference

pytestmark = pytest.mark.gpu

LOWEST = {W.BF16: float(torch.finfo(torch.bfloat16).min), W.F32: float(torch.finfo(torch.float32).min)}


@pytest.fixture(scope="module")
def F():
    import paper_2605_23163_amd as F
    F.load_library()
    return F


def close(got, ref, lse, n):
    r = (n / 256 + 64) * 2.0 ** -24
    with np.errstate(over="ignore"):
        fin = np.isfinite(ref.astype(np.float32))
    np.testing.assert_array_equal(got[~fin], np.full((~fin).sum(), -np.inf))
    assert np.isfinite(got[fin]).all()
    lse = np.broadcast_to(lse, ref.shape)[fin]
    tol = r * lse + 2.0 ** -22 * np.abs(ref[fin] + lse) + 2.0 ** -23 * np.abs(ref[fin]) + 1e-37
    assert (np.abs(got[fin] - ref[fin]) <= tol).all()


def rows_of(rng, V, dtype):
    low = LOWEST[dtype]
    rows = [np.full(V, low)]                                    # nothing but the lowest: every token has 1 / V
    rows.append(np.where(rng.random(V) < 0.5, low, -np.inf))
    rows[-1][V // 3] = low
    rows.append(np.where(np.arange(V) < 1, low, -np.inf))       # the lowest is all there is to choose
    rows.append(np.where(rng.random(V) < 0.5, low, low * 0.75))
    rows.append(np.where(np.arange(V) % 2, -low, low))          # the whole of the type's range
    for allowed in (1, 5, V // 2):
        for rest in (low, low * 0.77, (low, -np.inf)):
            x = np.full(V, rest) if np.isscalar(rest) else rng.choice(rest, V)
            at = rng.choice(V, allowed, replace=False)
            x[at] = 2.0 * rng.standard_normal(allowed)
            rows.append(x)
    x = np.full(V, low)                                         # allowed tokens next to one another
    x[V // 2:V // 2 + 5] = [0.0, 1.0, 1.0, -3.0, 0.5]
    rows.append(x)
    return W.to_storage(np.array([rows]), dtype)


@pytest.mark.parametrize("t", [0.3, 1.0, 2.5, 40.0])
@pytest.mark.parametrize("dtype", [W.BF16, W.F32])
@pytest.mark.parametrize("V", [10, 512, 4099, 16384, 40007, 152064])
def test_lowest_values(F, V, dtype, t):
    print_case(test="logprobs_lowest", V=V, dtype=dtype, t=t)
    rng = np.random.default_rng([V, 41])
    x = rows_of(rng, V, dtype)
    n, top = x.shape[1], min(8, V)
    f32t = float(1 / np.float32(1 / np.float32(t)))
    wide = W.widen(x, dtype).astype(np.float64)[0]
    for tokens in (np.zeros(n), np.full(n, V // 2 + 1), wide.argmax(1)):
        tokens = tokens.astype(np.int32)
        got = F.fdd_token_logprobs(to_dev(x), torch.from_numpy(tokens[None]).cuda(), top=top, temperature=t)
        lp, ent, ids, tlp = (g.cpu().numpy()[0] for g in got)
        rlp, rent, rids, rtlp, lse = reference(wide, tokens, top, f32t)
        close(lp.astype(np.float64), rlp, lse, V)
        np.testing.assert_array_equal(ids, rids)
        close(tlp.astype(np.float64), rtlp, lse[:, None], V)
        r = (V / 256 + 64) * 2.0 ** -24
        assert (np.abs(ent - rent) <= (2 * r + 2.0 ** -22) * rent + 1e-37).all()
    assert abs(float(lp[0]) + np.log(V)) <= 1e-5 * max(1.0, np.log(V))


@pytest.mark.parametrize("V,k", [(700, 700 // 2), (50001, 5), (152064, 1)])
def test_ruled_out_as_by_masked_fill(F, V, k):
    """Tokens ruled out by masked_fill with the type's lowest number score as tokens ruled out by -inf do."""
    print_case(test="logprobs_masked_fill", V=V, k=k)
    g = torch.Generator(device="cuda").manual_seed(V)
    for dt in (torch.bfloat16, torch.float32):
        x = torch.randn(2, 9, V, generator=g, device="cuda").to(dt)
        allowed = torch.zeros(V, dtype=torch.bool, device="cuda")
        allowed[torch.randperm(V, generator=g, device="cuda")[:k]] = True
        tokens = torch.nonzero(allowed)[0, 0].to(torch.int32).expand(2, 9).contiguous()
        a = F.fdd_token_logprobs(x.masked_fill(~allowed, torch.finfo(dt).min), tokens, top=1)
        b = F.fdd_token_logprobs(x.masked_fill(~allowed, -float("inf")), tokens, top=1)
        for s, t in zip(a, b):
            assert bool(torch.isfinite(s.float()).all()) and torch.equal(s, t)
