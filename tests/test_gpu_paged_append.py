"""Rows that join a paged cache, and what tokens of a tree see, on the GPU against plain references."""
import numpy as np
import pytest
import torch

import paper_2605_23163_amd as F
from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make_cache(g, N, page, max_pages, Hkv, D, dtype, lens, spare=2):
    pool = N * max_pages + spare
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    kv = [torch.randn(pool, Hkv, page, D, generator=g, device="cuda").to(DT[dtype]) for _ in range(2)]
    return F.PagedCache(*kv, order[:N * max_pages].view(N, max_pages).contiguous(), ints(lens))


def expected(cache, k, v, rows, n_rows, positions, rot):
    """Pools after the call, in float64, and the bound of K's."""
    kp, vp = (t.double().cpu().numpy().copy() for t in (cache.k, cache.v))
    bound = np.zeros_like(kp)
    table, lens = cache.page_table.cpu().numpy(), cache.lens.cpu().numpy()
    P, _, page, _ = kp.shape
    k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
    N, B = k.shape[:2]
    cap = table.shape[1] * page
    for n in range(N):
        for j in range(min(max(n_rows[n], 0), B)):
            src, slot = (j if rows is None else rows[n][j]), min(max(int(lens[n]), 0), cap) + j
            if not 0 <= src < B or slot >= cap:
                continue
            at = table[n, slot // page]
            if not 0 <= at < P:
                continue
            x, b = k[n, src], 0.0
            if rot is not None:
                w, m, inter, bf16 = rot
                pos = slot if positions is None else positions[n][src]
                y = R.rotate(x, np.array(pos), w, m, inter)
                b = R.rotate_bound(x, w, m, inter, bf16, y)
                x = y
            kp[at, :, slot % page], vp[at, :, slot % page] = x, v[n, src]
            bound[at, :, slot % page] = b
    return kp, vp, bound


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,B,page,max_pages,Hkv,D,lens,rot,with_rows,with_positions", [
    (1, 1, 16, 2, 1, 64, [0], None, False, False), (3, 1, 16, 4, 4, 128, [15, 16, 17], 128, False, False), (2, 5, 16, 3, 2, 64, [14, 30], 64, True, False),
    (3, 40, 32, 4, 4, 128, [0, 63, 100], 128, False, True), (2, 70, 64, 3, 3, 128, [1, 150], 24, True, True), (2, 33, 128, 2, 2, 64, [100, 0], 32, False, False),
    (4, 9, 1024, 1, 1, 128, [0, 1020, 1024, 5], 64, True, False), (2, 600, 64, 12, 2, 64, [3, 64], 64, False, False)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append(dtype, N, B, page, max_pages, Hkv, D, lens, rot, with_rows, with_positions, interleaved):
    g = torch.Generator(device="cuda").manual_seed(8)
    r = np.random.default_rng(9)
    cache = make_cache(g, N, page, max_pages, Hkv, D, dtype, lens)
    qkv = torch.randn(N, B, 5 * Hkv * D, generator=g, device="cuda").to(DT[dtype])      # parts of a wider projection
    k, v = (qkv[..., i * Hkv * D:(i + 1) * Hkv * D].unflatten(2, (Hkv, D)) for i in (1, 3))
    n_rows = [max(0, B - 2 * n) for n in range(N)] if N > 1 else [B]
    if N > 2:
        n_rows[2] = B + 7          # more than there are
    rows = r.integers(-2, B + 2, size=(N, B)).tolist() if with_rows else None
    positions = r.integers(-(1 << 31), (1 << 31) - 1, size=(N, B)).tolist() if with_positions else None
    table = w = None
    if rot:
        table = F.fdd_rope_table(rot, interleaved=interleaved)
        w = (*R.frequencies(rot, 1e4), interleaved, dtype == "bf16")
    cache.page_table[-1, -1] = -1                                # a page that is not there, and one that never was
    if max_pages > 1:
        cache.page_table[0, -1] = 1 << 30
    kp, vp, bound = expected(cache, k, v, rows, n_rows, positions, w)
    F.fdd_paged_append(k, v, cache, table=table, rows=None if rows is None else ints(rows), n_rows=ints(n_rows) if N > 1 else None,
                       positions=None if positions is None else ints(positions))
    assert torch.equal(cache.lens.cpu(), torch.tensor(lens, dtype=torch.int32))
    assert np.array_equal(cache.v.double().cpu().numpy(), vp)
    err = np.abs(cache.k.double().cpu().numpy() - kp)
    assert np.all(err <= bound), (err - bound).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_of_many_rows(dtype):
    """More than the caches hold: 34 MB written."""
    g = torch.Generator(device="cuda").manual_seed(10)
    B, Hkv, D = 4200 if dtype == "bf16" else 2100, 8, 128
    cache = make_cache(g, 2, 64, 70, Hkv, D, dtype, [30, 0])
    k, v = (torch.randn(2, B, Hkv, D, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    kp, vp, bound = expected(cache, k, v, None, [B, B - 100], None, (*R.frequencies(D, 1e4), False, dtype == "bf16"))
    F.fdd_paged_append(k, v, cache, table=F.fdd_rope_table(D), n_rows=ints([B, B - 100]))
    assert np.array_equal(cache.v.double().cpu().numpy(), vp)
    assert np.all(np.abs(cache.k.double().cpu().numpy() - kp) <= bound)


def test_append_into_a_pool_beyond_32_bits():
    page, Hkv, D = 1024, 8, 128
    pages = (1 << 32) // (page * Hkv * D) + 3                     # elements of a pool: more than 2^32
    k_pool, v_pool = (torch.zeros(pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = F.PagedCache(k_pool, v_pool, ints([[0, pages - 1]]), ints([page - 1]))
    k, v = (torch.randn(1, 2, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    F.fdd_paged_append(k, v, cache)
    for pool, x in ((k_pool, k), (v_pool, v)):
        assert torch.equal(pool[0, :, page - 1], x[0, 0]) and torch.equal(pool[pages - 1, :, 0], x[0, 1])
        assert int(torch.count_nonzero(pool[0]) + torch.count_nonzero(pool[pages - 1])) == int(torch.count_nonzero(x))
    # and attention reads it there
    now = cache._replace(lens=ints([page + 1]))
    q = torch.randn(1, 1, Hkv, D, device="cuda").bfloat16()
    out = F.fdd_paged_attn(q, now, k[:, :1], v[:, :1], max_len=page + 1)
    for h in range(Hkv):
        kk = torch.cat([k_pool[0, h], k_pool[pages - 1, h, :1], k[0, :1, h]]).double().cpu().numpy()
        vv = torch.cat([v_pool[0, h], v_pool[pages - 1, h, :1], v[0, :1, h]]).double().cpu().numpy()
        qq = q[0, :, h].double().cpu().numpy()
        want, a = R.attention(qq, kk, vv, np.ones((1, page + 2), dtype=bool), D ** -0.5)
        bound = R.attention_bound(qq, kk, D ** -0.5, want, a, True)
        assert np.all(np.abs(out[0, :, h].double().cpu().numpy() - want) <= bound)


@pytest.mark.parametrize("N,B", [(1, 1), (3, 2), (2, 16), (5, 63), (2, 64), (3, 65), (2, 128), (2, 200), (1, 256), (2, 300), (1, 512), (2, 777), (1, 1024)])
@pytest.mark.parametrize("kind", ["random", "chain", "star", "broken"])
def test_tree_mask(N, B, kind):
    r = np.random.default_rng(B)
    parents = np.zeros((N, B), dtype=np.int32)
    for i in range(B):
        parents[:, i] = {"random": r.integers(0, max(i, 1), size=N), "chain": i - 1, "star": 0, "broken": r.integers(-3, i + 4, size=N)}[kind]
    if kind == "broken":
        parents[0, 0] = 1 << 30
    lens = r.integers(0, 1 << 20, size=N).astype(np.int32)
    there = r.integers(0, B + 1, size=N).astype(np.int32)
    there[0] = B + 5 if N == 1 else B
    if N > 1:
        there[1] = 0
    mask, pos = F.fdd_tree_mask(ints(parents.tolist()), lens=ints(lens.tolist()), n_tokens=ints(there.tolist()))
    for n in range(N):
        c = min(int(there[n]), B)
        see = R.ancestors(parents[n], c)
        want = np.zeros((B, (B + 63) // 64), dtype=np.int64)
        want[:c] = R.pack_bits(see, B)
        assert np.array_equal(mask[n].cpu().numpy(), want)
        at = np.zeros(B, dtype=np.int64)
        at[:c] = lens[n] + see.sum(1) - 1
        assert np.array_equal(pos[n].cpu().numpy(), at)


def test_tree_mask_of_one_tree_for_all():
    parents = [-1, 0, 0, 1, 1, 2, 5]
    a = F.fdd_tree_mask(ints([parents] * 3), lens=ints([4, 5, 6]))
    for kw in (dict(lens=ints([4, 5, 6])), dict(lens=ints([4, 5, 6]), mask=torch.empty_like(a[0]), positions=torch.empty_like(a[1]))):
        b = F.fdd_tree_mask(ints(parents), **kw)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    m, p = F.fdd_tree_mask(ints(parents), N=2)
    assert m.shape == (2, 7, 1) and torch.equal(m[0], m[1]) and p[1].tolist() == [0, 1, 1, 2, 2, 2, 3]
    with pytest.raises(TypeError):
        F.fdd_tree_mask(ints([parents] * 3), lens=ints([4, 5]))
    with pytest.raises(F.FddError):
        F.fdd_tree_mask(torch.zeros(1, 1025, dtype=torch.int32, device="cuda"))
