"""Arguments of the calls on a paged cache, on rotary positions and on drafted trees: the native marshalling fills the structs that the
binding fills in Python, and leaves whatever is not the ordinary case to it."""
import ctypes as C

import pytest
import torch

import paper_2605_23163_amd as F
from paper_2605_23163_amd import binding as Bd
from paper_2605_23163_amd import paged as pg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    Bd.load_library()
    if pg._marshal() is None:
        pytest.skip("built without torch's headers")
    return pg._marshal()


class Recorder:
    """The library, except that calls do nothing and their structs are kept as bytes."""
    TYPES = {"fdd_rope": (pg.RopeParams,), "fdd_paged_append": (pg.PagedCacheStruct, pg.AppendParams), "fdd_tree_mask": (pg.TreeMaskParams,),
             "fdd_paged_attn": (pg.PagedCacheStruct, pg.PagedAttnParams), "fdd_tree_verify": (pg.TreeVerifyParams,)}

    def __init__(self, lib):
        self.lib, self.seen = lib, []

    def __getattr__(self, name):
        if name not in self.TYPES:
            return getattr(self.lib, name)

        def call(*a):
            for x, t in zip(a, self.TYPES[name]):
                p = t.from_buffer_copy(C.string_at(x, C.sizeof(t)))
                if name == "fdd_paged_append" and t is pg.AppendParams and p.rope:      # (a host struct beside the others)
                    self.seen.append(C.string_at(p.rope, C.sizeof(pg.RopeTableStruct)))
                    p.rope = 1
                self.seen.append(bytes(p))
            return 0
        return call


def structs(monkeypatch, native, call):
    lib, filled = Recorder(Bd.load_library()), []

    class Watched:
        def __getattr__(self, name):
            x = getattr(native, name)
            return x if isinstance(x, int) else lambda *a: filled.append(x(*a)) or filled[-1]
    with monkeypatch.context() as m:
        m.setattr(Bd, "_lib", lib)
        m.setattr(Bd, "_marshal", Watched() if native else None)
        call()
    return lib.seen, filled


def same(monkeypatch, M, call, ordinary=True):
    a, filled = structs(monkeypatch, M, call)
    b, _ = structs(monkeypatch, None, call)
    assert a and a == b and filled == [ordinary]


def z(*s, dtype=torch.bfloat16):
    return torch.zeros(s, dtype=dtype, device="cuda")


def i(*s):
    return z(*s, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope(monkeypatch, M, dtype):
    t = F.fdd_rope_table(48, interleaved=True, scaling="parts", stretch=2.0, original=100)
    q, k, p = z(2, 3, 6, 64, dtype=dtype), z(2, 3, 2, 64, dtype=dtype), i(2, 3)
    same(monkeypatch, M, lambda: F.fdd_rope(q, p, t, out=q))
    same(monkeypatch, M, lambda: F.fdd_rope(q, p, t, k, q, k, inverse=True))
    wide = z(2, 3, 10, 64, dtype=dtype)
    same(monkeypatch, M, lambda: F.fdd_rope(wide[:, :, :6], p, t, wide[:, :, 6:8], q, k))
    one = z(6, 64, dtype=dtype)
    same(monkeypatch, M, lambda: F.fdd_rope(one, i(), t, out=one))
    for wrong in (lambda: F.fdd_rope(q, p.long(), t, out=q), lambda: F.fdd_rope(q, p[:1], t, out=q), lambda: F.fdd_rope(q, p, t, k[..., :32], q, k[..., :32]),
                  lambda: F.fdd_rope(q, p, t, out=k), lambda: F.fdd_rope(q.transpose(2, 3), p, t, out=q.transpose(2, 3)),
                  lambda: F.fdd_rope(q[:1].expand(2, 3, 6, 64), p, t, out=q)):
        with pytest.raises((TypeError, ValueError)):
            structs(monkeypatch, M, wrong)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append(monkeypatch, M, dtype):
    t = F.fdd_rope_table(64)
    c = F.fdd_paged_cache(2, 5, 16, 3, 2, 64, dtype=dtype)
    k, v, l = z(2, 4, 2, 64, dtype=dtype), z(2, 4, 2, 64, dtype=dtype), i(2, 4)
    same(monkeypatch, M, lambda: F.fdd_paged_append(k, v, c))
    n = i(2)
    same(monkeypatch, M, lambda: F.fdd_paged_append(k, v, c, t, l, l, n))
    wide = z(2, 4, 6, 64, dtype=dtype)
    same(monkeypatch, M, lambda: F.fdd_paged_append(wide[:, :, :2], wide[:, :, 2:4], c, n_rows=n))
    for wrong in (lambda: F.fdd_paged_append(k[:1], v[:1], c), lambda: F.fdd_paged_append(k, v, c, rows=l[:, :2]), lambda: F.fdd_paged_append(k, v, c, n_rows=n.long()),
                  lambda: F.fdd_paged_append(k.half(), v.half(), c), lambda: F.fdd_paged_append(wide[:, :2, :2], v[:, :2].contiguous(), c)):
        with pytest.raises((TypeError, ValueError)):
            structs(monkeypatch, M, wrong)


def test_tree_mask(monkeypatch, M):
    mask, pos = z(2, 70, 2, dtype=torch.int64), i(2, 70)
    lens, n = i(2), i(2)
    per, one = i(2, 70), i(70)
    same(monkeypatch, M, lambda: F.fdd_tree_mask(per, lens, n, mask, pos))
    same(monkeypatch, M, lambda: F.fdd_tree_mask(one, None, n, mask, pos))
    same(monkeypatch, M, lambda: F.fdd_tree_mask(one, None, None, mask, pos))
    for wrong in (lambda: F.fdd_tree_mask(per, lens, n, mask[:, :, :1].contiguous(), pos), lambda: F.fdd_tree_mask(per, i(3), n, mask, pos)):
        with pytest.raises((TypeError, ValueError)):
            structs(monkeypatch, M, wrong)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention(monkeypatch, M, dtype):
    c = F.fdd_paged_cache(2, 5, 16, 3, 2, 64, dtype=dtype)
    q, k, v, n = z(2, 4, 6, 64, dtype=dtype), z(2, 4, 2, 64, dtype=dtype), z(2, 4, 2, 64, dtype=dtype), i(2)
    out, ws = torch.empty_like(q), z(1 << 22, dtype=torch.uint8)
    per, one = z(2, 4, 1, dtype=torch.int64), z(4, 1, dtype=torch.int64)
    same(monkeypatch, M, lambda: F.fdd_paged_attn(q, c, k, v, out=out, workspace=ws))
    same(monkeypatch, M, lambda: F.fdd_paged_attn(q, c, k, v, per, n, max_len=30, scale=0.3, out=out, workspace=ws))
    same(monkeypatch, M, lambda: F.fdd_paged_attn(q, c, k, v, one, n, out=out, workspace=ws))
    same(monkeypatch, M, lambda: F.fdd_paged_attn(q, c, k, v, causal_block=True, out=out, workspace=ws))
    wide = z(2, 4, 10, 64, dtype=dtype)
    same(monkeypatch, M, lambda: F.fdd_paged_attn(wide[:, :, :6], c, wide[:, :, 6:8], wide[:, :, 8:], n_tokens=n, out=out, workspace=ws))
    for wrong in (lambda: F.fdd_paged_attn(q, c, k[:, :2], v, out=out), lambda: F.fdd_paged_attn(q, c, k, v, per[:1], out=out), lambda: F.fdd_paged_attn(q, c, k, v, n_tokens=n[:1], out=out),
                  lambda: F.fdd_paged_attn(q, c, k, v, out=out[:, :2]), lambda: F.fdd_paged_attn(q[..., :32], c, k, v, out=out[..., :32])):
        with pytest.raises((TypeError, ValueError)):
            structs(monkeypatch, M, wrong)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_verify(monkeypatch, M, dtype):
    x, d, tok, u, par = z(2, 3, 50, dtype=dtype), z(2, 3, 50, dtype=dtype), i(2, 3), z(2, 3, 2, dtype=torch.float32), i(2, 3)
    outs = dict(path=i(2, 3), n_path=i(2), emitted=i(2, 3), chances=z(2, 3, dtype=torch.float32), workspace=z(1 << 16, dtype=torch.uint8))
    one, n = i(3), i(2)
    same(monkeypatch, M, lambda: F.fdd_tree_verify(x, tok, u, **outs))
    same(monkeypatch, M, lambda: F.fdd_tree_verify(x, tok, u, par, n_tokens=n, temperature=0.5, **outs))
    same(monkeypatch, M, lambda: F.fdd_tree_verify(x, tok, u, one, **outs))
    same(monkeypatch, M, lambda: F.fdd_tree_verify(x, tok, u, None, d, n, 0.7, 0.9, **outs))
    same(monkeypatch, M, lambda: F.fdd_tree_verify(x, tok, None, par, temperature=0, **outs))
    for wrong in (lambda: F.fdd_tree_verify(x, tok.long(), u, **outs), lambda: F.fdd_tree_verify(x, tok, u[..., 0], **outs), lambda: F.fdd_tree_verify(x, tok, u, None, d[:, :, :9], **outs),
                  lambda: F.fdd_tree_verify(x[:, :, ::2], tok, u, **outs), lambda: F.fdd_tree_verify(x, tok, u, one[:2], **outs)):
        with pytest.raises((TypeError, ValueError)):
            structs(monkeypatch, M, wrong)
