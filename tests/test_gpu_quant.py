"""The 8-bit prefix cache on the GPU: codes and scales bit for bit against the definition in 64 bits, rows read back exactly, and
attention over the cache against the fp64 oracle on the cache's values.

Tolerances of attention: the values of the cache are exact in the products, so they are those of fdd_block_attn.  bf16: ROW_TOL (see
gpu_util).  fp32: products of 2^-24 of their factors, sums over up to 2^13 keys and 128 channels, exponentials good to 2^-22: 1e-5 of a
row in norm is more than ten times what a row of average size takes."""
import numpy as np
import pytest
import torch

import fdd_workloads as W
from tests import quant_ref as Q
from tests.gpu_util import ROW_TOL, print_case, rand_attn, row_error, to_dev, to_f64

pytestmark = pytest.mark.gpu

TOL = {W.BF16: ROW_TOL, W.F32: 1e-5}


@pytest.fixture(scope="module")
def F():
    import paper_2605_23163_amd as F
    F.load_library()
    assert torch.cuda.is_available()
    return F


def poisoned(F, cap, Hkv, D):
    """A cache whose every byte is something else than a write leaves, and its host copy."""
    p = F.fdd_quant_prefix(cap, Hkv, D)
    for t in (p.k, p.v):
        t.view(torch.uint8).fill_(0xA5)
    for t in (p.k_scale, p.v_scale):
        t.fill_(-5.0)
    blocks = p.k_scale.shape[1]
    host = [np.full((Hkv, blocks * 64, D), 0xA5, np.uint8) for _ in range(2)] + [np.full((Hkv, blocks), -5.0) for _ in range(2)]
    return p, host


def same(p, host):
    for t, h in zip(p, host):
        if t.dtype == torch.float8_e4m3fn:
            nan = lambda c: np.where(c & 127 == 127, 127, c)        # (a NaN has no sign)
            np.testing.assert_array_equal(nan(t.view(torch.uint8).cpu().numpy()), nan(h))
        else:
            np.testing.assert_array_equal(t.cpu().numpy().astype(np.float64), h)


def values(rng, n, Hkv, D, dtype, special):
    """Rows whose spread changes from row to row; with `special` also zeros, ties, tiny, huge, infinite and missing values."""
    x = rng.standard_normal((n, Hkv, D)) * np.exp2(rng.integers(-6, 7, size=(n, 1, 1)))
    if special and n:
        x[rng.random(x.shape) < 0.1] = 0.0
        at = rng.random(x.shape) < 0.1
        x[at] = Q.VALUES[rng.integers(0, 127, size=int(at.sum()))] * rng.choice([1.0, 1.0625, 0.9375, -1.0], size=int(at.sum()))
        flat = x.reshape(-1)
        flat[rng.integers(0, flat.size, 3)] = [np.inf, -np.inf, np.nan]
        flat[rng.integers(0, flat.size, 2)] = [1e-38, 2.0 ** -112]
        if n > 200:
            x[:64] = 0.0
            x[64:128] = np.finfo(np.float32).max * rng.choice([1.0, -0.5], size=x[64:128].shape)
            x[128:192] *= 2.0 ** -120
    st = W.to_storage(x, dtype)
    return st, W.widen(st, dtype)


@pytest.mark.parametrize("dtype", [W.BF16, W.F32])
@pytest.mark.parametrize("Hkv,D", [(1, 64), (3, 128), (2, 64)])
@pytest.mark.parametrize("row0,n", [(0, 1), (0, 64), (0, 333), (5, 58), (5, 60), (63, 1), (64, 65), (130, 0), (191, 200)])
def test_codes_and_scales(F, dtype, Hkv, D, row0, n):
    print_case(test="quantize", dtype=dtype, Hkv=Hkv, D=D, row0=row0, n=n)
    rng = np.random.default_rng([row0, n, Hkv, D])
    p, host = poisoned(F, 448, Hkv, D)
    for at, m, special in ((0, row0, False), (row0, n, True)):
        st = [values(rng, m, Hkv, D, dtype, special) for _ in range(2)]
        assert F.fdd_prefix_quantize(*(to_dev(s) for s, _ in st), p, row0=at) == at + m
        for j in range(2):
            Q.write(host[j], host[2 + j], st[j][1], at)
    torch.cuda.synchronize()
    same(p, host)
    lo = max(0, row0 - 7)
    for dt, out in ((W.BF16, torch.bfloat16), (W.F32, torch.float32)):
        k, v = F.fdd_prefix_dequantize(p, row0 + n - lo, row0=lo, dtype=out)
        for j, t in enumerate((k, v)):
            assert t.dtype == out and t.shape == (row0 + n - lo, Hkv, D)
            np.testing.assert_array_equal(to_f64(t), Q.read(host[j], host[2 + j], lo, row0 + n - lo))


def test_rows_join_in_pieces(F):
    """A cache grows block by block, its rows larger and larger: every scale grows, and what was there moves with it."""
    print_case(test="append")
    rng = np.random.default_rng(9)
    p, host = poisoned(F, 1000, 2, 128)
    held = 0
    for i, n in enumerate((1, 2, 40, 21, 100, 3, 64, 129, 7, 1, 300)):
        st = W.to_storage(rng.standard_normal((n, 2, 128)) * 2.0 ** (i % 4 * 3), W.BF16)
        x = to_dev(st)
        held = F.fdd_prefix_quantize(x, -x, p, row0=held)
        for j, sign in enumerate((1, -1)):
            Q.write(host[j], host[2 + j], sign * W.widen(st, W.BF16), held - n)
        same(p, host)
    assert held == 668
    # an earlier row0 gives up what lay behind; the block's scale stays at least as it was
    x = to_dev(W.to_storage(np.full((3, 2, 128), 2.0 ** -9), W.BF16))
    assert F.fdd_prefix_quantize(x, x, p, row0=70) == 73
    for j in range(2):
        Q.write(host[j], host[2 + j], np.full((3, 2, 128), 2.0 ** -9), 70)
    same(p, host)


def test_rows_may_lie_apart(F):
    print_case(test="strided_rows")
    rng = np.random.default_rng(10)
    Hkv, D, n = 2, 64, 150
    for dtype in (W.BF16, W.F32):
        qkv = to_dev(W.to_storage(rng.standard_normal((n, 8 + 2 * Hkv, D)), dtype))       # a fused projection
        k, v = qkv[:, 8:8 + Hkv], qkv[:, 8 + Hkv:]
        a, b = F.fdd_quant_prefix(n, Hkv, D), F.fdd_quant_prefix(n, Hkv, D)
        F.fdd_prefix_quantize(k, v, a)
        F.fdd_prefix_quantize(k.contiguous(), v.contiguous(), b)
        for s, t in zip(a[:2], b[:2]):
            assert torch.equal(s[:, :n].view(torch.uint8), t[:, :n].view(torch.uint8))
        wide = torch.full((n, 3 * Hkv, D), 7.0, dtype=torch.float32, device="cuda")
        F.fdd_prefix_dequantize(a, n, k=wide[:, :Hkv], v=wide[:, 2 * Hkv:])
        ref = F.fdd_prefix_dequantize(b, n, dtype=torch.float32)
        assert torch.equal(wide[:, :Hkv], ref[0]) and torch.equal(wide[:, 2 * Hkv:], ref[1]) and bool((wide[:, Hkv:2 * Hkv] == 7).all())
        one = F.fdd_prefix_dequantize(a, 1, row0=77)
        assert torch.equal(one[0].float(), ref[0][77:78])
    with pytest.raises(ValueError, match="contiguous"):
        F.fdd_prefix_quantize(k.transpose(1, 2).contiguous().transpose(1, 2), v, a)
    with pytest.raises(ValueError, match="overlap"):
        F.fdd_prefix_quantize(k[:1].expand(5, Hkv, D), v[:1].expand(5, Hkv, D), a)
    odd = torch.zeros(10 * (Hkv * D + 4), dtype=torch.bfloat16, device="cuda").as_strided((10, Hkv, D), (Hkv * D + 4, D, 1))
    with pytest.raises(F.FddError, match="multiple of 16"):
        F.fdd_prefix_quantize(odd, odd, a)


# ---- attention ---------------------------------------------------------------------------------------------------------------

def cached(F, d, dtype, cap=None, extra=0):
    """The prefix rows of d in a cache, and d with the cache's values in their place (in the storage type: they are exact)."""
    L, Hkv, D = d["prefix_k"].shape
    p, host = poisoned(F, (L if cap is None else cap) + extra, Hkv, D) if L or cap or extra else (None, None)
    if L:
        F.fdd_prefix_quantize(to_dev(d["prefix_k"]), to_dev(d["prefix_v"]), p)
        d = dict(d)
        for j, name in enumerate(("prefix_k", "prefix_v")):
            Q.write(host[j], host[2 + j], W.widen(d[name], dtype), 0)
            d[name] = W.to_storage(Q.read(host[j], host[2 + j], 0, L), dtype)
    return p, d


def check(F, oracle, d, dtype, scale=None, causal=False, ext=None, E=0, positions=None, **kw):
    p, d = cached(F, d, dtype, extra=kw.pop("extra", 0))
    ek, ev = ext if ext is not None else (None, None)
    dev = {k: to_dev(v) for k, v in d.items()}
    if ext is not None:
        kw.update(ext_k=to_dev(ek), ext_v=to_dev(ev), E=E)
    if positions is not None:
        kw.update(q_positions=torch.tensor(positions, dtype=torch.int32, device="cuda"), out=torch.full_like(dev["q"], 3.0))
    out = F.fdd_block_attn_quant(dev["q"], p, d["prefix_k"].shape[0], dev["block_k"], dev["block_v"], scale=scale, causal_block=causal, **kw)
    got = to_f64(out)
    ref = oracle.block_attn(d["q"], d["prefix_k"], d["prefix_v"], d["block_k"], d["block_v"], scale=scale, causal_block=causal, ext_k=ek, ext_v=ev, E=E)
    if positions is not None:
        left = np.ones(got.shape[:2], bool)
        left.reshape(-1)[list(positions)] = False
        assert (got[left] == 3.0).all()
        got, ref = got[~left], ref[~left]
    assert np.isfinite(got).all()
    err = row_error(got, ref)
    assert err <= TOL[dtype], f"row error {err}"
    return dev, p, out


SHAPES = [
    # N, B,  L,   Hq, Hkv, D
    (1, 8, 256, 4, 1, 64),
    (1, 1, 1, 4, 2, 64),          # one key, one query
    (1, 1, 77, 4, 2, 128),
    (1, 4, 63, 7, 1, 128),
    (1, 4, 64, 7, 1, 64),
    (2, 5, 65, 6, 2, 128),
    (2, 5, 130, 6, 2, 128),
    (3, 20, 333, 14, 2, 128),     # 420 stacked rows: rollouts straddle wavefronts and M-tiles
    (5, 32, 1000, 28, 4, 128),
    (2, 70, 64, 8, 8, 64),        # more block keys than a tile
    (4, 16, 0, 4, 2, 128),        # no prefix at all
    (9, 3, 200, 3, 1, 64),        # many tiny rollouts inside one wavefront tile
    (1, 32, 2048, 28, 4, 128),
    (1, 32, 5000, 28, 4, 64),
    (8, 32, 1500, 28, 4, 128),
]


@pytest.mark.parametrize("dtype", [W.BF16, W.F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_matches_oracle(F, oracle, shape, dtype):
    N, B, L, Hq, Hkv, D = shape
    print_case(test="quant_attn", shape=shape, dtype=dtype)
    d = rand_attn(np.random.default_rng(list(shape)), *shape, dtype)
    check(F, oracle, d, dtype)


@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7, 64])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_extension_causal_positions(F, oracle, D, splits):
    print_case(test="quant_attn_forms", D=D, splits=splits)
    rng = np.random.default_rng([D, splits])
    N, B, L, Hq, Hkv, E, cap = 4, 24, 700, 14, 2, 37, 61
    for dtype in (W.BF16, W.F32):
        d = rand_attn(rng, N, B, L, Hq, Hkv, D, dtype)
        ext = [W.to_storage(rng.standard_normal((N, cap, Hkv, D)), dtype) for _ in range(2)]
        positions = sorted(rng.choice(N * B, size=31, replace=False).tolist())
        check(F, oracle, d, dtype, splits=splits, causal=True, extra=200)
        check(F, oracle, d, dtype, splits=splits, ext=ext, E=E)
        check(F, oracle, d, dtype, splits=splits, ext=ext, E=E, causal=True, positions=positions, scale=0.3)
        check(F, oracle, d, dtype, splits=splits, positions=[95])


@pytest.mark.parametrize("N,L,Hq,Hkv,D", [(16, 700, 28, 4, 128), (40, 333, 14, 2, 64), (3, 9000, 28, 4, 128), (12, 4100, 16, 2, 128)])
def test_attention_of_many_rows(F, oracle, N, L, Hq, Hkv, D):
    """Several M-tiles of 128 and of 256 rows a head, pieces and ranges."""
    print_case(test="quant_attn_rows", N=N, L=L, Hq=Hq, Hkv=Hkv, D=D)
    check(F, oracle, rand_attn(np.random.default_rng([N, L]), N, 32, L, Hq, Hkv, D, W.BF16), W.BF16)


@pytest.mark.parametrize("spread", [2.0 ** -100, 2.0 ** -20, 2.0 ** 20])
def test_scales_of_blocks_differ(F, oracle, spread):
    """Every block and head has a scale of its own, K and V do too; the values of V take the result's range with them."""
    print_case(test="quant_attn_scales", spread=spread)
    rng = np.random.default_rng(21)
    d = rand_attn(rng, 2, 8, 400, 8, 2, 128, W.BF16)
    f = {k: W.widen(v, W.BF16) for k, v in d.items()}
    f["prefix_k"] *= np.exp2(rng.integers(-3, 2, size=(7, 2))).repeat(64, 0)[:400, :, None]
    f["prefix_v"] *= np.exp2(rng.integers(-6, 6, size=(7, 2))).repeat(64, 0)[:400, :, None] * spread
    f["block_v"] *= spread
    check(F, oracle, {k: W.to_storage(v, W.BF16) for k, v in f.items()}, W.BF16)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,splits", [(1, 1), (1, 2), (4, 1), (4, 3)])
def test_long_runs_of_tiles(F, oracle, D, N, splits):
    """One workgroup walks 203 tiles (more than the ring of scales holds), 102 or 68, every tile with scales of its own; M-tiles of 128
    rows (N = 1) and of 256."""
    print_case(test="quant_attn_long", D=D, N=N, splits=splits)
    rng = np.random.default_rng([D, N, splits])
    B, L, Hq, Hkv = 32, 64 * 202 + 17, 24, 4
    d = rand_attn(rng, N, B, L, Hq, Hkv, D, W.BF16)
    f = {k: W.widen(d[k], W.BF16) for k in ("prefix_k", "prefix_v")}
    f["prefix_k"] *= np.exp2(rng.integers(-2, 2, size=(203, Hkv))).repeat(64, 0)[:L, :, None]
    f["prefix_v"] *= np.exp2(rng.integers(-3, 4, size=(203, Hkv))).repeat(64, 0)[:L, :, None]
    d.update({k: W.to_storage(v, W.BF16) for k, v in f.items()})
    p, d = cached(F, d, W.BF16)
    dev = {k: to_dev(v) for k, v in d.items()}
    out = to_f64(F.fdd_block_attn_quant(dev["q"], p, L, dev["block_k"], dev["block_v"], splits=splits))
    rows = np.stack([rng.integers(0, n, 48) for n in (N, B, Hq)], axis=1)
    ref = oracle.block_attn(d["q"], d["prefix_k"], d["prefix_v"], d["block_k"], d["block_v"], rows=rows)
    assert row_error(out[tuple(rows.T)], ref) <= ROW_TOL


@pytest.mark.parametrize("spread", [0, 100, -80])
@pytest.mark.parametrize("D,N", [(64, 1), (128, 1), (128, 12)])
def test_segments_that_cancel(F, D, N, spread):
    """Two pieces of the keys whose averages nearly cancel.  Scores are all 0, so that every probability is 1 and an output is the mean of
    n values: fp32 sums n 2^-24 of the largest one; a piece's averages in 11 bits of the largest one, 2^-11 of it at most; the
    output in bf16, 2^-8 of itself.  (Averages in bf16 would be off by 2^-9 of themselves and more.)"""
    print_case(test="quant_attn_cancel", D=D, N=N, spread=spread)
    rng = np.random.default_rng([D, N, spread + 100])
    B, L, Hq, Hkv = 8, 512, 8, 2
    d = rand_attn(rng, N, B, L, Hq, Hkv, D, W.BF16)
    v = rng.uniform(1.0, 2.0, (L, Hkv, D))
    v[L // 2:] *= -1.0
    d["prefix_v"] = W.to_storage(np.ldexp(v, spread), W.BF16)
    d["block_v"] = W.to_storage(np.ldexp(rng.uniform(-1.0, 1.0, (N, B, Hkv, D)), spread), W.BF16)
    p, d = cached(F, d, W.BF16)
    dev = {k: to_dev(x) for k, x in d.items()}
    out = to_f64(F.fdd_block_attn_quant(torch.zeros_like(dev["q"]), p, L, dev["block_k"], dev["block_v"], splits=2))
    pv, bv = (W.widen(d[k], W.BF16).astype(np.float64) for k in ("prefix_v", "block_v"))
    ref = (pv.sum(0) + bv.sum(1, keepdims=True)) / (L + B)                 # [N,1,Hkv,D], one for all queries
    ref = np.repeat(ref, Hq // Hkv, axis=2)
    top = np.abs(pv).max()
    assert (np.abs(out - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + (L + B) * 2.0 ** -24) * top).all()


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_random_shapes(F, oracle, seed):
    """Shapes that the cases above do not list, every form of the call among them."""
    rng = np.random.default_rng([seed, 77])
    for case in range(24):
        dtype = W.BF16 if case % 4 else W.F32
        D, Hkv, G = int(rng.choice([64, 128])), int(rng.choice([1, 2, 4, 8])), int(rng.choice([1, 2, 3, 7]))
        N, B = int(rng.integers(1, 20)), int(rng.choice([1, 2, 5, 16, 31, 32, 33, 40, 64, 65, 100]))
        L = int(rng.choice([0, 1, 63, 64, 65, 127, 128, 200, 777, 1024, 1500, 4096, 5000]))
        E = int(rng.choice([0, 0, 1, 7, 64, 90]))
        if N * B * Hkv * G * (L + E + B) * D > (2e8 if dtype == W.F32 else 2e9):
            N, L = max(1, N // 5), min(L, 1500)
        kw = dict(causal=bool(rng.integers(0, 2)), splits=int(rng.choice([0, 0, 0, 1, 2, 3, 5, 9])), extra=int(rng.choice([0, 0, 130])))
        if E:
            cap = E + int(rng.integers(0, 5))
            kw.update(E=E, ext=[W.to_storage(rng.standard_normal((N, cap, Hkv, D)), dtype) for _ in range(2)])
        if rng.integers(0, 3) == 0:
            keep = rng.random(N * B) < rng.choice([0.1, 0.5, 0.9])
            keep[rng.integers(N * B)] = True
            kw["positions"] = np.flatnonzero(keep).tolist()
        print_case(test="quant_attn_sweep", seed=seed, case=case, dtype=dtype, N=N, B=B, L=L, Hq=Hkv * G, Hkv=Hkv, D=D, E=E, causal=kw["causal"],
                   splits=kw["splits"], listed="positions" in kw)
        check(F, oracle, rand_attn(rng, N, B, L, Hkv * G, Hkv, D, dtype), dtype, **kw)


def test_rows_behind_the_prefix_are_not_used(F):
    """A cache holds more rows than the call says, NaN among them: the result is that of a cache that ends there."""
    print_case(test="quant_attn_behind")
    rng = np.random.default_rng(22)
    for L, D in ((100, 64), (128, 128), (701, 128)):
        d = rand_attn(rng, 2, 16, L, 8, 2, D, W.BF16)
        p, _ = cached(F, d, W.BF16, cap=L + 300)
        dev = {k: to_dev(v) for k, v in d.items()}
        a = F.fdd_block_attn_quant(dev["q"], p, L, dev["block_k"], dev["block_v"])
        for t in p[:2]:
            t[:, L:].view(torch.uint8).fill_(0x7F)
        for t in p[2:]:
            t[:, (L + 63) // 64:] = float("nan")
        b = F.fdd_block_attn_quant(dev["q"], p, L, dev["block_k"], dev["block_v"])
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())


@pytest.mark.parametrize("dtype", [W.BF16, W.F32])
def test_same_as_attention_on_the_rows_read_back(F, dtype):
    print_case(test="quant_attn_plain", dtype=dtype)
    rng = np.random.default_rng(23)
    for N, B, L, Hq, Hkv, D in ((2, 32, 1000, 28, 4, 128), (1, 8, 2500, 8, 8, 64), (16, 32, 600, 28, 4, 128)):
        d = rand_attn(rng, N, B, L, Hq, Hkv, D, dtype)
        p, _ = cached(F, d, dtype)
        dev = {k: to_dev(v) for k, v in d.items()}
        k, v = F.fdd_prefix_dequantize(p, L, dtype=dev["q"].dtype)
        a = F.fdd_block_attn_quant(dev["q"], p, L, dev["block_k"], dev["block_v"])
        b = F.fdd_block_attn(dev["q"], k, v, dev["block_k"], dev["block_v"])
        assert row_error(to_f64(a), to_f64(b)) <= TOL[dtype]


@pytest.mark.parametrize("dtype", [W.BF16, W.F32])
@pytest.mark.parametrize("D,L", [(64, 500), (128, 1111), (128, 64)])
def test_batch(F, dtype, D, L):
    print_case(test="quant_attn_batch", dtype=dtype, D=D, L=L)
    rng = np.random.default_rng([D, L])
    P, N, B, Hq, Hkv, E = 3, 2, 8, 8, 2, 10
    ds = [rand_attn(rng, N, B, L, Hq, Hkv, D, dtype) for _ in range(P)]
    # problems lie apart: the batch is a slice of a larger one
    cap = (L + 63) // 64 * 64 + 64
    big = F.fdd_quant_prefix(cap, Hkv, D, batch=2 * P)
    for t in big[:2]:
        t.view(torch.uint8).fill_(0x7F)
    for t in big[2:]:
        t.fill_(float("nan"))
    sub = F.QuantPrefix(*(t[::2] for t in big))
    one = lambda i: F.QuantPrefix(*(t[i] for t in sub))
    for i, d in enumerate(ds):
        F.fdd_prefix_quantize(to_dev(d["prefix_k"]), to_dev(d["prefix_v"]), one(i))
    dev = {k: torch.stack([to_dev(d[k]) for d in ds]) for k in ("q", "block_k", "block_v")}
    ek, ev = (to_dev(W.to_storage(rng.standard_normal((P, N, E + 2, Hkv, D)), dtype)) for _ in range(2))
    for kw in ({}, dict(causal_block=True, ext_k=ek, ext_v=ev, E=E)):
        need = F.fdd_block_attn_quant_batched_workspace(dev["q"], sub, L, dev["block_k"], dev["block_v"], **{k: v for k, v in kw.items() if k != "causal_block"})
        ws = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
        out = F.fdd_block_attn_quant_batched(dev["q"], sub, L, dev["block_k"], dev["block_v"], workspace=ws, **kw)
        for i in range(P):
            kwi = dict(kw, ext_k=ek[i], ext_v=ev[i]) if kw else {}
            ref = F.fdd_block_attn_quant(dev["q"][i], one(i), L, dev["block_k"][i], dev["block_v"][i], **kwi)
            assert row_error(to_f64(out[i]), to_f64(ref)) <= TOL[dtype]


def test_no_positions(F):
    d = {k: to_dev(v) for k, v in rand_attn(np.random.default_rng(3), 1, 4, 0, 4, 2, 64, W.BF16).items()}
    out = torch.full_like(d["q"], 2.0)
    F.fdd_block_attn_quant(d["q"], None, 0, d["block_k"], d["block_v"], out=out, q_positions=torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert bool((out == 2.0).all())


def test_positions_out_of_range_or_order(F):
    """The host cannot read the list: such entries lead nowhere outside the arrays, and the other rows stay as they were."""
    print_case(test="quant_positions")
    d = {k: to_dev(v) for k, v in rand_attn(np.random.default_rng(4), 6, 16, 300, 8, 2, 128, W.BF16).items()}
    p = F.fdd_quant_prefix(300, 2, 128)
    F.fdd_prefix_quantize(d["prefix_k"], d["prefix_v"], p)
    for pos in ([-5, 3, 95, 96, 2 ** 31 - 1], [90, 3, 50, 3], [7] * 20):
        out = torch.full_like(d["q"], 2.0)
        F.fdd_block_attn_quant(d["q"], p, 300, d["block_k"], d["block_v"], out=out, q_positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        named = sorted({min(max(x, 0), 95) for x in pos})
        rest = [i for i in range(96) if i not in named]
        assert bool((out.view(96, 8, 128)[rest] == 2.0).all())


# ---- as they are used: together, on other streams, in a graph ----------------------------------------------------------------------

def test_step_over_a_growing_cache_in_a_graph(F):
    """A block is attended to over the cache, joins it, its tokens are scored, and the next block attends to the longer cache: recorded
    once, every replay gives the eager result."""
    print_case(test="quant_graph")
    rng = np.random.default_rng(31)
    N, B, L, Hq, Hkv, D, V = 2, 16, 150, 8, 2, 128, 5000
    d = {k: to_dev(v) for k, v in rand_attn(rng, N, B, L, Hq, Hkv, D, W.BF16).items()}
    logits = to_dev(W.to_storage(rng.standard_normal((N, B, V)) * 3, W.BF16))
    tokens = torch.from_numpy(rng.integers(0, V, (N, B)).astype(np.int32)).cuda()
    prompt = F.fdd_quant_prefix(L + B, Hkv, D)
    for t in prompt:
        t.view(torch.uint8).fill_(0)
    F.fdd_prefix_quantize(d["prefix_k"], d["prefix_v"], prompt)
    p = F.QuantPrefix(*(torch.empty_like(t) for t in prompt))
    out, out2 = torch.empty_like(d["q"]), torch.empty_like(d["q"])
    back = [torch.empty((L + B, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    f = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="cuda")
    lp = (f(N, B), f(N, B), f(N, B, 5, dtype=torch.int32), f(N, B, 5))
    need = max(F.fdd_block_attn_quant_workspace(d["q"], p, n, d["block_k"], d["block_v"]) for n in (L, L + B))
    ws = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    ws_l = torch.empty(max(256, F.fdd_token_logprobs_workspace(logits, top=5)), dtype=torch.uint8, device="cuda")

    def step():
        for s, t in zip(prompt, p):
            t.view(torch.uint8).copy_(s.view(torch.uint8))
        F.fdd_block_attn_quant(d["q"], p, L, d["block_k"], d["block_v"], out=out, workspace=ws)
        F.fdd_token_logprobs(logits, tokens, top=5, logprobs=lp[0], entropy=lp[1], top_ids=lp[2], top_logprobs=lp[3], workspace=ws_l)
        held = F.fdd_prefix_quantize(d["block_k"][0], d["block_v"][0], p, row0=L)
        F.fdd_block_attn_quant(d["q"], p, held, d["block_k"], d["block_v"], out=out2, workspace=ws)
        F.fdd_prefix_dequantize(p, held, k=back[0], v=back[1])

    results = (out, out2, *back, *lp, *p)

    def scrub():
        for t in results:
            t.view(torch.uint8).fill_(0x55)
        torch.cuda.synchronize()

    step()
    torch.cuda.synchronize()
    eager = [t.view(torch.uint8).clone() for t in results]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        scrub()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(results, eager)):
            assert torch.equal(a.view(torch.uint8), b), f"result {i} differs from the eager run"


def test_on_another_stream(F):
    print_case(test="quant_stream")
    rng = np.random.default_rng(32)
    d = {k: to_dev(v) for k, v in rand_attn(rng, 2, 16, 900, 8, 2, 64, W.BF16).items()}
    logits = to_dev(W.to_storage(rng.standard_normal((2, 16, 3001)), W.F32))
    tokens = torch.zeros(2, 16, dtype=torch.int32, device="cuda")
    mask = torch.ones(2, 16, dtype=torch.uint8, device="cuda")

    def go(p, **kw):
        F.fdd_prefix_quantize(d["prefix_k"], d["prefix_v"], p, **kw)
        return (F.fdd_block_attn_quant(d["q"], p, 900, d["block_k"], d["block_v"], **kw), *F.fdd_prefix_dequantize(p, 900, **kw),
                *F.fdd_token_logprobs(logits, tokens, mask=mask, top=3, **kw))

    ref = go(F.fdd_quant_prefix(900, 2, 64))
    p = F.fdd_quant_prefix(900, 2, 64)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = go(p, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(ref, got):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_far_end_of_a_large_cache(F):
    """Codes whose place passes 32 bits: 4.1e9 of them an array."""
    print_case(test="quant_far")
    Hkv, D, cap = 64, 128, 64 * 7900
    p = F.fdd_quant_prefix(cap, Hkv, D)
    assert p.k.numel() > 2 ** 32 - 2 ** 28 and (Hkv - 1) * cap * D > 2 ** 31
    x = torch.randn(70, Hkv, D, dtype=torch.bfloat16, device="cuda")
    for t in p[2:]:
        t.fill_(2.0 ** -117)        # (no rows in front of the first one written)
    F.fdd_prefix_quantize(x, -x, p, row0=cap - 70)
    small = F.fdd_quant_prefix(128, Hkv, D)
    for t in small[2:]:
        t.fill_(2.0 ** -117)
    F.fdd_prefix_quantize(x, -x, small, row0=58)
    a, b = F.fdd_prefix_dequantize(p, 70, row0=cap - 70), F.fdd_prefix_dequantize(small, 70, row0=58)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # attention over the head of every head's rows, among them the last head's, 4e9 codes on
    y = torch.randn(100, Hkv, D, dtype=torch.bfloat16, device="cuda")
    q, bk = torch.randn(1, 4, Hkv, D, dtype=torch.bfloat16, device="cuda"), torch.randn(1, 4, Hkv, D, dtype=torch.bfloat16, device="cuda")
    F.fdd_prefix_quantize(y, y, p)
    F.fdd_prefix_quantize(y, y, small)
    assert torch.equal(F.fdd_block_attn_quant(q, p, 100, bk, bk), F.fdd_block_attn_quant(q, small, 100, bk, bk))
