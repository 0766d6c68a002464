"""fdd_token_logprobs against softmax in 64 bits.

Errors that are counted: a sum of n terms in fp32, n / 256 of them one after the other and the rest in a tree or in fp64, is good to
r = (n / 256 + 64) 2^-24, the 64 for the tree, for 2^x (2^-22) and for its argument, of magnitude up to 30 where a term counts.
ln(1 + S) <= S / (1 + S) * (its own size) turns r into r ln(1 + S) at most; the difference to the largest logit and its division by
the temperature are good to 2^-23, and the result is rounded once, 2^-24.  So |error| <= r ln(1 + S) + 2^-22 |y| + 2^-24 |result|; the
entropy, ln(1 + S) - U / (1 + S) with both terms >= 0, is good to 2 r + 2^-22 of itself."""
import numpy as np
import pytest
import torch

import fdd_workloads as W
from tests.gpu_util import print_case, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    import paper_2605_23163_amd as F
    F.load_library()
    return F


def reference(x, tokens, top, t):
    """x [rows,V] float64"""
    V = x.shape[1]
    ids = np.argsort(-x, axis=1, kind="stable")[:, :top]
    m = x.max(1)
    at = x.argmax(1)
    with np.errstate(invalid="ignore"):
        y = (x - m[:, None]) / t
    e = np.exp(y)
    e[np.arange(len(x)), at] = 0.0
    lse = np.log1p(e.sum(1))
    logp = y - lse[:, None]
    p = np.exp(logp)
    ent = -np.sum(p * np.where(p > 0, logp, 0.0), axis=1)
    known = (tokens >= 0) & (tokens < V)
    lp = np.where(known, logp[np.arange(len(x)), np.where(known, tokens, 0)], -np.inf)
    return lp, ent, ids, np.take_along_axis(logp, ids, 1), lse


def close(got, ref, lse, n):
    r = (n / 256 + 64) * 2.0 ** -24
    fin = np.isfinite(ref)
    np.testing.assert_array_equal(got[~fin], ref[~fin])
    lse = np.broadcast_to(lse, ref.shape)
    tol = r * lse + 2.0 ** -22 * np.abs(ref + lse) + 2.0 ** -23 * np.abs(ref) + 1e-37
    assert (np.abs(got - ref)[fin] <= tol[fin]).all(), float((np.abs(got - ref)[fin] / tol[fin]).max())


def check(F, x, tokens, dtype, top, t=1.0, mask=None, **kw):
    """x [N,B,V] storage"""
    N, B, V = x.shape
    m = None if mask is None else torch.from_numpy(mask).cuda()
    got = F.fdd_token_logprobs(to_dev(x), torch.from_numpy(tokens).cuda(), mask=m, top=top, temperature=t, **kw)
    lp, ent, ids, tlp = (g.cpu().numpy() for g in got)
    assert lp.shape == (N, B) and ids.shape == tlp.shape == (N, B, top)
    sel = np.ones(N * B, bool) if mask is None else mask.reshape(-1) == 1
    f32t = float(1 / np.float32(1 / np.float32(t)))       # (what is divided by is good to 2^-24: counted with y)
    rlp, rent, rids, rtlp, lse = reference(W.widen(x, dtype).reshape(N * B, V)[sel], tokens.reshape(-1)[sel], top, f32t)
    close(lp.reshape(-1)[sel].astype(np.float64), rlp, lse, V)
    np.testing.assert_array_equal(ids.reshape(N * B, top)[sel], rids)
    if top:
        close(tlp.reshape(N * B, top)[sel].astype(np.float64), rtlp, lse[:, None], V)
    r = (V / 256 + 64) * 2.0 ** -24
    err = np.abs(ent.reshape(-1)[sel] - rent)
    assert (err <= (2 * r + 2.0 ** -22) * rent + 1e-37).all()
    if mask is not None:
        assert (lp.reshape(-1)[~sel] == 0).all() and (ids.reshape(N * B, top)[~sel] == -1).all()
    return got


def logits(rng, N, B, V, dtype, std=2.0):
    x = rng.standard_normal((N, B, V)) * std
    hit = rng.random((N, B)) < 0.4
    n, b = np.nonzero(hit)
    x[n, b, rng.integers(0, V, size=len(n))] += 14.0
    return W.to_storage(x, dtype)


@pytest.mark.parametrize("dtype", [W.BF16, W.F32])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 255, 511, 512, 513, 1000, 4095, 4097, 9973, 16384, 16391, 32768, 50001, 152064, 262147])
def test_matches_reference(F, V, dtype):
    rng = np.random.default_rng(V)
    for N, B, top, t in ((1, 1, 1, 1.0), (3, 5, 5, 0.7), (2, 3, 32, 1.3), (1, 4, 0, 1.0)):
        top = min(top, V)
        print_case(test="logprobs", V=V, dtype=dtype, N=N, B=B, top=top)
        x = logits(rng, N, B, V, dtype)
        tokens = rng.integers(0, V, size=(N, B)).astype(np.int32)
        check(F, x, tokens, dtype, top, t)


@pytest.mark.parametrize("dtype", [W.BF16, W.F32])
@pytest.mark.parametrize("V", [40, 3001, 40007])
def test_ties_order_and_missing_entries(F, V, dtype):
    print_case(test="logprobs_ties", V=V, dtype=dtype)
    rng = np.random.default_rng([V, 1])
    top = min(32, V)
    rows = [np.zeros(V), np.full(V, -3.0), np.arange(V) * 1.0, -np.arange(V) * 1.0, rng.integers(0, 3, V) * 1.0, np.where(np.arange(V) % 2, 0.0, -0.0)]
    few = np.full(V, -np.inf)
    few[rng.integers(0, V, 5)] = rng.standard_normal(5)
    last = np.full(V, -np.inf)
    last[V - 1] = 3.0
    sure = rng.standard_normal(V)
    sure[V // 2] = 60.0
    near = np.full(V, -30.0)
    near[1] = 1e-3
    big = rng.standard_normal(V) * 3e37
    x = W.to_storage(np.array([rows + [few, last, sure, near, big]]), dtype)
    B = x.shape[1]
    for tokens in (np.zeros((1, B)), np.full((1, B), V - 1), np.full((1, B), V // 2), np.full((1, B), -1), np.full((1, B), V), np.full((1, B), 2 ** 31 - 1)):
        check(F, x, tokens.astype(np.int32), dtype, top)


@pytest.mark.parametrize("dtype", [W.BF16, W.F32])
@pytest.mark.parametrize("V", [9001, 15000, 100000])
def test_largest_entries_in_few_places(F, V, dtype):
    """Rows whose largest entries repeat with a period: a few threads of a workgroup have them all."""
    print_case(test="logprobs_few_places", V=V, dtype=dtype)
    rng = np.random.default_rng([V, 2])
    per = 16 // (2 if dtype == W.BF16 else 4) * 64
    x = rng.standard_normal((1, 6, V))
    for b, share in enumerate((1, 8, 30, 31, 33, 64)):
        x[0, b] += 20.0 * ((np.arange(V) % per) < per // 64 * share)
    for top in (1, 5, 32):
        check(F, W.to_storage(x, dtype), np.zeros((1, 6), np.int32), dtype, top)


def test_a_row_without_entries(F):
    print_case(test="logprobs_empty")
    for V in (5, 700, 40000):
        x = torch.full((1, 3, V), -float("inf"), device="cuda")
        x[0, 1, 2] = 0.0
        lp, ent, ids, tlp = F.fdd_token_logprobs(x, torch.tensor([[2, 2, -1]], dtype=torch.int32, device="cuda"), top=3)
        assert bool(torch.isnan(lp[0, 0])) and float(lp[0, 1]) == 0.0 and float(lp[0, 2]) == -float("inf")
        assert bool(torch.isnan(ent[0, 0])) and float(ent[0, 1]) == 0.0
        assert ids[0, 0].tolist() == [0, 1, 2] and bool(torch.isnan(tlp[0, 0]).all())
        assert ids[0, 1].tolist() == [2, 0, 1] and tlp[0, 1].tolist() == [0.0, -float("inf"), -float("inf")]


@pytest.mark.parametrize("V", [300, 20001])
def test_selected_rows_only(F, V):
    print_case(test="logprobs_mask", V=V)
    rng = np.random.default_rng(V)
    N, B = 4, 33
    x = logits(rng, N, B, V, W.BF16)
    tokens = rng.integers(0, V, size=(N, B)).astype(np.int32)
    for mask in ((rng.random((N, B)) < 0.4).astype(np.uint8), np.zeros((N, B), np.uint8), np.eye(N, B, dtype=np.uint8)):
        check(F, x, tokens, W.BF16, 4, mask=mask)
    # what the caller had in the outputs of the others stays, and their logits are not read
    mask = np.zeros((N, B), np.uint8)
    mask[1, 5] = 1
    mask[2, 6] = 2          # (only 1 selects)
    lp, ent = torch.full((N, B), 7.0, device="cuda"), torch.full((N, B), 8.0, device="cuda")
    ids, tlp = torch.full((N, B, 4), 9, dtype=torch.int32, device="cuda"), torch.full((N, B, 4), 10.0, device="cuda")
    F.fdd_token_logprobs(to_dev(x), torch.from_numpy(tokens).cuda(), mask=torch.from_numpy(mask).cuda(), top=4, logprobs=lp, entropy=ent, top_ids=ids, top_logprobs=tlp)
    for t, was in ((lp, 7.0), (ent, 8.0), (ids, 9), (tlp, 10.0)):
        same = (t == was).reshape(N, B, -1).all(-1).cpu().numpy()
        assert not same[1, 5] and same.sum() == N * B - 1


def test_many_rows(F):
    print_case(test="logprobs_rows")
    rng = np.random.default_rng(5)
    for N, B, V, dtype in ((64, 70, 500, W.F32), (16, 32, 9000, W.BF16), (300, 8, 130, W.BF16)):
        x = logits(rng, N, B, V, dtype)
        check(F, x, rng.integers(0, V, size=(N, B)).astype(np.int32), dtype, 6)


def test_twice_the_same(F):
    """The joins run in a fixed order: two calls agree bit for bit."""
    print_case(test="logprobs_repeat")
    rng = np.random.default_rng(6)
    x = to_dev(logits(rng, 8, 32, 152064 // 4, W.BF16))
    tokens = torch.from_numpy(rng.integers(0, 30000, (8, 32)).astype(np.int32)).cuda()
    a = F.fdd_token_logprobs(x, tokens, top=20)
    for _ in range(3):
        for s, t in zip(a, F.fdd_token_logprobs(x, tokens, top=20)):
            assert torch.equal(s.view(torch.int32), t.view(torch.int32))


def test_against_differences(F):
    """The gradient of the entropy along a direction, and what the log probabilities of all tokens add up to."""
    print_case(test="logprobs_sum")
    rng = np.random.default_rng(7)
    V = 24
    x = torch.from_numpy(rng.standard_normal((1, 1, V)).astype(np.float32)).cuda()
    every = x.expand(1, V, V).contiguous()
    lp, ent, ids, tlp = F.fdd_token_logprobs(every, torch.arange(V, dtype=torch.int32, device="cuda")[None], top=V)
    p = torch.exp(lp.double())
    assert abs(float(p.sum()) - 1) < 1e-6 and abs(float(-(p * lp).sum()) - float(ent[0, 0])) < 1e-6
    assert torch.equal(tlp[0, 0], lp[0, ids[0, 0].long()])


def test_unaligned_workspace_and_missing_outputs(F):
    import ctypes as C
    from paper_2605_23163_amd import binding as bd
    print_case(test="logprobs_outputs")
    rng = np.random.default_rng(8)
    V = 30000
    x = to_dev(logits(rng, 2, 3, V, W.BF16))
    tok = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    ref = F.fdd_token_logprobs(x, tok, top=4)
    lib = F.load_library()
    ws = torch.empty(max(256, F.fdd_token_logprobs_workspace(x, top=4)), dtype=torch.uint8, device="cuda")
    for names in (("logprobs",), ("entropy",), ("top_ids", "top_logprobs"), ("entropy", "logprobs")):
        p = bd._logprob_params(x, 4, 1.0)
        p.logits, p.tokens = x.data_ptr(), tok.data_ptr() if "logprobs" in names else None
        p.workspace, p.workspace_bytes, p.stream = ws.data_ptr(), ws.numel(), bd._stream_ptr(None)
        outs = {n: torch.empty_like(t) for n, t in zip(("logprobs", "entropy", "top_ids", "top_logprobs"), ref) if n in names}
        for n, t in outs.items():
            setattr(p, n, t.data_ptr())
        assert lib.fdd_token_logprobs(C.byref(p)) == 0, F.fdd_last_error()
        for n, t in zip(("logprobs", "entropy", "top_ids", "top_logprobs"), ref):
            if n in outs:
                assert torch.equal(outs[n].view(torch.int32), t.view(torch.int32))


@pytest.mark.parametrize("seed", [1, 2, 3, 4])
def test_random_calls(F, seed):
    """Sizes, types, selected positions and values drawn: few or many entries that can be chosen, few different values, large offsets."""
    rng = np.random.default_rng([77, seed])
    for i in range(16):
        N, B = int(rng.integers(1, 9)), int(rng.integers(1, 41))
        V = int(np.exp(rng.uniform(0, np.log(60000))))
        V = max(1, min(V, 2000000 // (N * B)))
        dtype, top = (W.BF16, W.F32)[rng.integers(2)], int(rng.integers(0, min(V, 32) + 1))
        kind, t = int(rng.integers(0, 4)), float(rng.choice([1.0, 0.3, 2.5, 40.0]))
        print_case(test="logprobs_random", seed=seed, i=i, N=N, B=B, V=V, dtype=dtype, top=top, kind=kind, t=t)
        x = W.widen(logits(rng, N, B, V, dtype), dtype).astype(np.float64)
        if kind == 1:
            x[rng.random(x.shape) < rng.choice([0.5, 0.99])] = -np.inf
            np.put_along_axis(x, rng.integers(0, V, (N, B, 1)), 1.0, 2)
        elif kind == 2:
            x = np.rint(x * 0.5)
        elif kind == 3:
            x[..., : V // 3] += 20.0
            x -= 100.0
        mask = None if rng.random() < 0.4 else (rng.random((N, B)) < rng.choice([0.1, 0.5, 1.0])).astype(np.uint8)
        tokens = rng.integers(-1, V + 1, (N, B)).astype(np.int32)
        check(F, W.to_storage(x, dtype), tokens, dtype, top, t=t, mask=mask)
