"""Refusals of the calls on a paged cache, on rotary positions and on trees of drafted tokens, and the frequencies' table: host code
only, nothing is launched (no GPU is needed)."""
import ctypes as C
import os

import numpy as np
import pytest

from paper_2605_23163_amd import binding as bd
from paper_2605_23163_amd import paged as pg
from tests import paged_ref as R


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(bd.library_path()):
        from paper_2605_23163_amd import build
        build.build()
    return bd.load_library()


def filled(t, base, kw):
    p = t()
    for values in (base, kw):
        for k, v in values.items():
            if isinstance(v, dict):
                for a, b in v.items():
                    setattr(getattr(p, k), a, b)
            else:
                setattr(p, k, v)
    return p


BIG = 1 << 46
CACHE = dict(k=BIG, v=2 * BIG, page_table=256, lens=512, N=4, pages=100, page_size=64, max_pages=32, Hkv=4, D=128, dtype=1)
TABLE = dict(turns=1024, rot_dim=128, interleaved=0, magnitude=1.0)


def cache(**kw):
    return filled(pg.PagedCacheStruct, CACHE, kw)


BAD_CACHES = [(dict(N=0), 2), (dict(pages=-1), 2), (dict(max_pages=0), 2), (dict(Hkv=0), 2), (dict(page_size=8), 4), (dict(page_size=48), 4),
              (dict(page_size=2048), 4), (dict(D=96), 4), (dict(dtype=5), 3), (dict(max_pages=1 << 24), 2), (dict(N=1 << 20, Hkv=1 << 9, D=64), 2),
              (dict(Hkv=1 << 17), 2), (dict(pages=1 << 30, Hkv=8), 2), (dict(Hkv=32768, page_size=1024), 2), (dict(reserved=1), 4), (dict(k=None), 1),
              (dict(v=None), 1), (dict(page_table=None), 1), (dict(lens=None), 1), (dict(k=BIG + 8), 4), (dict(lens=514), 4)]


# ---- the frequencies ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rot_dim,base,scaling,stretch,original", [
    (128, 1e6, None, 1.0, None), (64, 1e4, None, 1.0, None), (2, 1e4, None, 1.0, None), (128, 1e6, "linear", 4.0, None), (24, 1e4, "base", 8.0, None),
    (4, 1e4, "base", 2.0, None), (128, 1e6, "parts", 4.0, 32768), (64, 1e4, "parts", 10.0, 4096), (1024, 5e5, "parts", 1.0, 100), (128, 1e4, "linear", 1.0, None)])
def test_turns(lib, rot_dim, base, scaling, stretch, original):
    p = pg.RopeScaling(rot_dim, pg._SCALINGS[scaling], base, stretch, original or 1.0)
    turns, magnitude = (C.c_uint64 * (rot_dim // 2))(), C.c_float()
    assert lib.fdd_rope_turns(C.byref(p), turns, C.byref(magnitude)) == 0
    w, m = R.frequencies(rot_dim, base, scaling, stretch, original)
    want = w / R.TWO_PI * np.longdouble(2) ** 64
    got = np.array(list(turns), dtype=np.uint64).astype(np.longdouble)
    # (extended precision: 2^-64 of itself for each of a dozen operations, and half a unit of the rounding)
    assert np.all(np.abs(got - want) <= 0.5 + want * np.longdouble(2) ** -58)
    assert abs(magnitude.value - m) <= 2.0 ** -24 * m


@pytest.mark.parametrize("kw,code", [(dict(rot_dim=0), 2), (dict(rot_dim=7), 2), (dict(rot_dim=1026), 2), (dict(scaling=4), 4), (dict(scaling=-1), 4), (dict(base=1.0), 4),
                                     (dict(base=float("nan")), 4), (dict(base=float("inf")), 4), (dict(scaling=1, stretch=0.5), 4), (dict(scaling=1, stretch=float("inf")), 4),
                                     (dict(scaling=3, original=0.0), 4), (dict(scaling=3, original=float("nan")), 4), (dict(scaling=2, rot_dim=2), 2),
                                     (dict(scaling=2, base=1e300, stretch=1e300), 4)])
def test_turns_refusals(lib, kw, code):
    p = filled(pg.RopeScaling, dict(rot_dim=64, scaling=0, base=1e4, stretch=2.0, original=100.0), kw)
    turns, magnitude = (C.c_uint64 * 1024)(), C.c_float()
    assert lib.fdd_rope_turns(C.byref(p), turns, C.byref(magnitude)) == code
    assert lib.fdd_last_error().decode().startswith("fdd_rope_turns:")
    assert lib.fdd_rope_turns(None, turns, C.byref(magnitude)) == 1
    assert lib.fdd_rope_turns(C.byref(p), None, C.byref(magnitude)) == 1


# ---- refusals ------------------------------------------------------------------------------------------------------------

def rope(**kw):
    return filled(pg.RopeParams, dict(rows=32, Hq=28, Hk=4, D=128, dtype=1, table=TABLE, positions=2048, q=BIG, q_out=2 * BIG, k=3 * BIG, k_out=4 * BIG), kw)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), 2), (dict(Hq=0), 2), (dict(D=0), 2), (dict(D=2048), 2), (dict(Hk=0), 2), (dict(dtype=2), 3), (dict(flags=2), 4), (dict(Hq=65535, Hk=2), 2),
    (dict(q=None), 1), (dict(q_out=None), 1), (dict(positions=None), 1), (dict(k=None), 1), (dict(k_out=None), 1), (dict(q_stride=100), 2), (dict(k_stride=1 << 29), 2),
    (dict(q=BIG + 1), 4), (dict(positions=2050), 4), (dict(q_out=BIG + 2), 4), (dict(k_out=BIG), 4), (dict(q_out=2048), 4), (dict(k_out=1024), 4),
    (dict(q_out=BIG, q_out_stride=28 * 128 + 8), 4), (dict(rows=1 << 30), 2), (dict(table=dict(turns=None)), 1), (dict(table=dict(rot_dim=130)), 2), (dict(table=dict(rot_dim=63)), 2),
    (dict(table=dict(rot_dim=0)), 2), (dict(table=dict(interleaved=2)), 4), (dict(table=dict(magnitude=float("nan"))), 4), (dict(table=dict(reserved=1)), 4),
    (dict(table=dict(turns=1028)), 4)])
def test_rope_refusals(lib, kw, code):
    assert lib.fdd_rope(C.byref(rope(**kw))) == code
    assert lib.fdd_last_error().decode().startswith("fdd_rope:")
    assert lib.fdd_rope(None) == 1


def test_rope_of_no_rows(lib):
    assert lib.fdd_rope(C.byref(rope(rows=0, q=None, q_out=None, positions=None))) == 0


def append(**kw):
    return filled(pg.AppendParams, dict(B=32, k=3 * BIG, v=4 * BIG), kw)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_paged_cache_refusals(lib, kw, code):
    c = cache(**kw)
    assert lib.fdd_paged_append(C.byref(c), C.byref(append())) == code
    assert lib.fdd_last_error().decode().startswith("fdd_paged_append:")
    assert lib.fdd_paged_attn(C.byref(c), C.byref(attn())) == code
    assert lib.fdd_last_error().decode().startswith("fdd_paged_attn:")
    assert lib.fdd_paged_attn_workspace(C.byref(c), C.byref(attn())) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), 2), (dict(reserved=3), 4), (dict(k=None), 1), (dict(v=None), 1), (dict(k=3 * BIG + 8), 4), (dict(rows=6), 4), (dict(positions=2), 4), (dict(n_rows=1), 4),
    (dict(k_stride=64), 2), (dict(v_stride=4 * 128 + 4), 2), (dict(B=1 << 29), 2), (dict(k=BIG + 4096), 4), (dict(v=2 * BIG), 4), (dict(rows=BIG), 4), (dict(n_rows=BIG), 4)])
def test_append_refusals(lib, kw, code):
    assert lib.fdd_paged_append(C.byref(cache()), C.byref(append(**kw))) == code
    assert lib.fdd_last_error().decode().startswith("fdd_paged_append:")


def test_append_refuses_what_overlaps(lib):
    assert lib.fdd_paged_append(C.byref(cache(v=BIG + 4096)), C.byref(append())) == 4
    assert lib.fdd_paged_append(C.byref(cache(lens=BIG)), C.byref(append())) == 4
    t = filled(pg.RopeTableStruct, TABLE, dict(rot_dim=256))
    assert lib.fdd_paged_append(C.byref(cache()), C.byref(append(rope=C.addressof(t)))) == 2
    assert lib.fdd_paged_append(None, C.byref(append())) == 1 and lib.fdd_paged_append(C.byref(cache()), None) == 1


def tree(**kw):
    return filled(pg.TreeMaskParams, dict(N=4, B=32, parents=256, mask=4096, positions=8192), kw)


@pytest.mark.parametrize("kw,code", [(dict(N=0), 2), (dict(B=0), 2), (dict(B=1025), 4), (dict(parents=None), 1), (dict(mask=None, positions=None), 1), (dict(parents_stride=31), 2),
                                     (dict(parents_stride=-32), 2), (dict(parents=258), 4), (dict(mask=4100), 4), (dict(positions=8194), 4), (dict(lens=3), 4), (dict(n_tokens=3), 4),
                                     (dict(N=1 << 22, B=1), 2), (dict(positions=256), 4), (dict(positions=4096 + 1016), 4), (dict(mask=256 + 120), 4), (dict(lens=8192 + 8), 4),
                                     (dict(n_tokens=4096 + 1020), 4)])
def test_tree_mask_refusals(lib, kw, code):
    assert lib.fdd_tree_mask(C.byref(tree(**kw))) == code
    assert lib.fdd_last_error().decode().startswith("fdd_tree_mask:")
    assert lib.fdd_tree_mask(None) == 1


def attn(**kw):
    return filled(pg.PagedAttnParams, dict(B=32, Hq=28, q=3 * BIG, block_k=4 * BIG, block_v=5 * BIG, out=6 * BIG, workspace=7 * BIG, workspace_bytes=1 << 45), kw)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), 2), (dict(Hq=0), 2), (dict(Hq=30), 2), (dict(max_len=-1), 2), (dict(flags=2), 4), (dict(reserved=1), 4), (dict(scale=float("nan")), 4), (dict(scale=float("inf")), 4),
    (dict(B=1 << 25), 2), (dict(B=1 << 23, Hq=128), 2), (dict(q=None), 1), (dict(block_k=None), 1), (dict(block_v=None), 1), (dict(out=None), 1), (dict(q=3 * BIG + 8), 4), (dict(mask=4), 4), (dict(n_tokens=2), 4),
    (dict(mask=4096, flags=1), 4), (dict(q_stride=128), 2), (dict(k_stride=4 * 128 + 2), 2), (dict(v_stride=1 << 24), 2), (dict(mask=4096, mask_stride=5), 2), (dict(out=3 * BIG), 4),
    (dict(out=BIG), 4), (dict(workspace=None), 5), (dict(workspace=7 * BIG + 128), 5), (dict(workspace_bytes=1000), 5),
    (dict(mask=6 * BIG), 4), (dict(n_tokens=6 * BIG + 64), 4), (dict(workspace=6 * BIG), 4), (dict(workspace=4 * BIG), 4), (dict(mask=7 * BIG), 4),
    (dict(mask=4096, mask_stride=1 << 55), 2), (dict(B=1 << 18, Hq=128), 2)])
def test_attn_refusals(lib, kw, code):
    assert lib.fdd_paged_attn(C.byref(cache()), C.byref(attn(**kw))) == code
    assert lib.fdd_last_error().decode().startswith("fdd_paged_attn:")
    assert lib.fdd_paged_attn(None, C.byref(attn())) == 1 and lib.fdd_paged_attn(C.byref(cache()), None) == 1


def test_attn_workspace(lib):
    size = lambda c, **kw: lib.fdd_paged_attn_workspace(C.byref(c), C.byref(attn(**kw)))
    assert size(cache()) > 0 and size(cache()) % 256 == 0
    assert size(cache(), Hq=30) == 0
    assert size(cache(max_pages=1), B=1) == 0                     # one tile of the cache, one of the tokens: never cut
    assert size(cache(), max_len=64, B=1) == 0
    assert size(cache(), max_len=1 << 30) == size(cache())


def verify(**kw):
    return filled(pg.TreeVerifyParams, dict(N=4, B=32, V=50001, dtype=1, temperature=1.0, draft_temperature=1.0, logits=BIG, tokens=256, uniforms=4096, path=8192, n_path=12288,
                                            emitted=16384, workspace=2 * BIG, workspace_bytes=1 << 45), kw)


@pytest.mark.parametrize("kw,code", [
    (dict(N=0), 2), (dict(B=-1), 2), (dict(V=0), 2), (dict(V=1 << 31), 2), (dict(B=1025), 4), (dict(N=1 << 20), 2), (dict(dtype=9), 3), (dict(reserved=1), 4), (dict(temperature=-1.0), 4),
    (dict(temperature=float("nan")), 4), (dict(temperature=float("inf")), 4), (dict(temperature=1e-9), 4), (dict(draft_logits=3 * BIG, draft_temperature=0.0), 4), (dict(logits=None), 1),
    (dict(tokens=None), 1), (dict(uniforms=None), 1), (dict(path=None), 1), (dict(n_path=None), 1), (dict(emitted=None), 1), (dict(draft_logits=3 * BIG, parents=256), 4),
    (dict(parents=256, parents_stride=16), 2), (dict(logits=BIG + 1), 4), (dict(tokens=258), 4), (dict(chances=2), 4), (dict(workspace=None), 5), (dict(workspace=2 * BIG + 8), 5),
    (dict(workspace_bytes=64), 5), (dict(V=(1 << 30) + 1), 2), (dict(N=1 << 22, B=1, V=8), 2), (dict(N=1 << 20, B=1, V=1 << 20), 2), (dict(N=1 << 14, B=1024), 2),
    (dict(path=256), 4), (dict(emitted=256 + 508), 4), (dict(n_path=8192 + 4), 4), (dict(chances=16384), 4), (dict(chances=4096 + 1020), 4), (dict(workspace=BIG), 4),
    (dict(emitted=2 * BIG), 4), (dict(parents=8192), 4), (dict(n_tokens=12288), 4),
    # (with temperature 0 draft_logits have no part: the call gets as far as its workspace)
    (dict(draft_logits=3 * BIG, parents=256, temperature=0.0, draft_temperature=0.0, workspace=None), 5)])
def test_verify_refusals(lib, kw, code):
    assert lib.fdd_tree_verify(C.byref(verify(**kw))) == code
    assert lib.fdd_last_error().decode().startswith("fdd_tree_verify:")
    assert lib.fdd_tree_verify(None) == 1


def test_verify_workspace(lib):
    size = lambda **kw: lib.fdd_tree_verify_workspace(C.byref(verify(**kw)))
    assert size() > 0 and size() % 256 == 0 and size(V=0) == 0
    assert size(temperature=0.0) == size()
    assert size(draft_logits=3 * BIG) >= size()


# ---- the binding's own checks, on tensors that are not on a GPU ------------------------------------------------------------

def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    import paper_2605_23163_amd as F
    table = F.fdd_rope_table(64, device="cpu")
    assert table.turns.shape == (32,) and table.turns.dtype == torch.int64 and table.magnitude == 1.0
    q = torch.zeros(2, 3, 4, 64)
    with pytest.raises(ValueError):
        F.fdd_rope(q, torch.zeros(2, 3, dtype=torch.int32), table)
    with pytest.raises(TypeError):
        F.fdd_rope(q, torch.zeros(2, 3, dtype=torch.int64), table)
    with pytest.raises(ValueError):
        F.fdd_rope(q, torch.zeros(2, 3, dtype=torch.int32), table, k_out=q)
    cache = F.fdd_paged_cache(2, 5, 16, 3, 2, 64, dtype=torch.float32, device="cpu")
    assert cache.k.shape == (5, 2, 16, 64) and bool((cache.page_table == -1).all()) and bool((cache.lens == 0).all())
    k = torch.zeros(2, 3, 2, 64)
    with pytest.raises(ValueError):
        F.fdd_paged_append(k, k, cache)
    with pytest.raises(ValueError):
        F.fdd_paged_attn(q, cache, k, k)
    with pytest.raises(ValueError):
        F.fdd_tree_mask(torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        F.fdd_tree_verify(torch.zeros(2, 3, 10), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, 2))


@pytest.mark.parametrize("kw", [dict(rot_dim=7), dict(rot_dim=64, scaling="linear", stretch=0.0), dict(rot_dim=64, base=0.5)])
def test_rope_table_refusals(kw):
    pytest.importorskip("torch")
    import paper_2605_23163_amd as F
    with pytest.raises(F.FddError):
        F.fdd_rope_table(device="cpu", **kw)
    with pytest.raises(ValueError):
        F.fdd_rope_table(64, scaling="parts", stretch=2.0, device="cpu")
    with pytest.raises(ValueError):
        F.fdd_rope_table(64, scaling="other", device="cpu")
