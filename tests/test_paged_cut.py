"""The cut of fdd_paged_attn's keys: every tile once, no more pieces than the workspace has room for, and a place for each that the merge finds.
Host arithmetic, nothing is launched."""
import ctypes as C
import os
import random

import pytest

from paper_2605_23163_amd import binding as bd
from paper_2605_23163_amd import paged as pg
from tests import paged_cut as cut


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(bd.library_path()):
        from paper_2605_23163_amd import build
        build.build()
    return bd.load_library()


def workspace(lib, N, B, Hq, Hkv, D, bf16, page, max_pages, max_len):
    big = 1 << 40
    c = pg.PagedCacheStruct(k=big, v=big, page_table=256, lens=256, N=N, pages=8, page_size=page, max_pages=max_pages, Hkv=Hkv, D=D, dtype=1 if bf16 else 0)
    p = pg.PagedAttnParams(B=B, Hq=Hq, max_len=max_len, q=big, block_k=big, block_v=big, out=big)
    return lib.fdd_paged_attn_workspace(C.byref(c), C.byref(p))


@pytest.mark.parametrize("seed", range(60))
def test_every_tile_once(lib, seed):
    r = random.Random(seed)
    bf16, D, page = r.random() < 0.6, r.choice((64, 128)), r.choice((16, 64, 256))
    Hkv = r.choice((1, 2, 4, 8))
    Hq, B, N = Hkv * r.choice((1, 4, 7)), r.choice((1, 2, 5, 21, 32, 64, 65, 128, 200, 700)), r.choice((1, 2, 3, 5, 9, 12, 20, 33, 70, 130))
    max_pages = r.choice((1, 4, 40, 300))
    capacity = page * max_pages
    max_len = r.choice((0, 0, capacity // 2 + 1))
    lens = [r.choice((0, 1, capacity, r.randrange(capacity + 1))) for _ in range(N)]
    counts = [r.choice((0, B, r.randrange(B + 1))) for _ in range(N)]
    items = cut.items(lens, counts, B, Hq, Hkv, bf16, capacity, max_len)
    waves, used, kt, W, most, partials = cut.plan(N, B, Hq, Hkv, bf16, capacity, max_len)
    assert len(items) <= most
    need = workspace(lib, N, B, Hq, Hkv, D, bf16, page, max_pages, max_len)
    rows = most * used * 32 if partials else 0
    assert need == cut.ceil(rows * D * (2 if bf16 else 4), 256) * 256 + cut.ceil(rows * 16, 256) * 256
    if not partials:
        assert all(i.pieces == 1 for i in items)
    seen = {}
    for at, i in enumerate(items):
        seen.setdefault((i.n, i.kh, i.mt), []).append((i.piece, i.t_begin, i.t_end, i.pieces))
        assert cut.joined_at(lens, counts, B, Hq, Hkv, bf16, capacity, i.n, i.kh, i.mt, i.piece, max_len) == at
    cached = [min(L, max_len or capacity) for L in lens]
    mtiles = {n: cut.ceil(counts[n] * (Hq // Hkv), waves * 32) for n in range(N)}
    assert set(seen) == {(n, kh, mt) for n in range(N) for kh in range(Hkv) for mt in range(mtiles[n])}
    for (n, _, _), pieces in seen.items():
        pieces.sort()
        assert [p[0] for p in pieces] == list(range(pieces[0][3]))
        assert pieces[0][1] == 0 and pieces[-1][2] == cut.ceil(cached[n], kt) + cut.ceil(counts[n], kt)
        assert all(a[2] == b[1] for a, b in zip(pieces, pieces[1:])) and all(p[2] > p[1] for p in pieces)
