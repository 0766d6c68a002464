"""Arguments of the calls on an 8-bit cache and on log probabilities: the native marshalling fills the structs that the binding
fills in Python, and leaves whatever is not the ordinary case to it."""
import ctypes as C

import pytest
import torch

from paper_2605_23163_amd import binding as Bd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    Bd.load_library()
    if Bd._marshal is None:
        pytest.skip("built without torch's headers")
    return Bd._marshal


class Recorder:
    """The library, except that calls do nothing and their structs are kept as bytes."""
    SIZES = {"fdd_prefix_quantize": (C.sizeof(Bd.QuantCache), None, C.sizeof(Bd.QuantRows)), "fdd_block_attn_quant": (C.sizeof(Bd.AttnParams), C.sizeof(Bd.QuantCache)),
             "fdd_token_logprobs": (C.sizeof(Bd.LogprobParams),)}
    SIZES["fdd_prefix_dequantize"] = SIZES["fdd_prefix_quantize"]

    def __init__(self, lib):
        self.lib, self.seen = lib, []

    def __getattr__(self, name):
        if name not in self.SIZES:
            return getattr(self.lib, name)

        def call(*a):
            self.seen.append([x if n is None else C.string_at(x, n) for x, n in zip(a, self.SIZES[name])] + list(a[len(self.SIZES[name]):]))
            return 0
        return call


def structs(monkeypatch, native, call):
    """What the library is given, and whether the native module filled it."""
    lib = Recorder(Bd.load_library())
    filled = []

    class Watched:
        def __getattr__(self, name):
            return lambda *a: filled.append(getattr(native, name)(*a)) or filled[-1]
    with monkeypatch.context() as m:
        m.setattr(Bd, "_lib", lib)
        m.setattr(Bd, "_marshal", Watched() if native else None)
        call()
    return lib.seen, filled


def same(monkeypatch, M, call, ordinary=True):
    a, filled = structs(monkeypatch, M, call)
    b, _ = structs(monkeypatch, None, call)
    assert a == b and filled == [ordinary]


def z(*s, dtype=torch.bfloat16):
    return torch.zeros(s, dtype=dtype, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows(monkeypatch, M, dtype):
    p = Bd.fdd_quant_prefix(200, 3, 64)
    k, v = z(20, 3, 64, dtype=dtype), z(20, 3, 64, dtype=dtype)
    same(monkeypatch, M, lambda: Bd.fdd_prefix_quantize(k, v, p, row0=7))
    same(monkeypatch, M, lambda: Bd.fdd_prefix_quantize(k[:0], v[:0], p))
    same(monkeypatch, M, lambda: Bd.fdd_prefix_dequantize(p, 20, k=k, v=v))
    wide = z(20, 9, 64, dtype=dtype)
    seen, filled = structs(monkeypatch, M, lambda: Bd.fdd_prefix_quantize(wide[:, :3], wide[:, 3:6], p))
    assert filled == [False] and len(seen) == 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention(monkeypatch, M, dtype):
    N, B, Hq, Hkv, D, L = 2, 5, 6, 3, 64, 150
    p = Bd.fdd_quant_prefix(L, Hkv, D)
    q, bk, bv = z(N, B, Hq, D, dtype=dtype), z(N, B, Hkv, D, dtype=dtype), z(N, B, Hkv, D, dtype=dtype)
    out, ws = torch.empty_like(q), z(1 << 20, dtype=torch.uint8)
    ek, ev = z(N, 9, Hkv, D, dtype=dtype), z(N, 9, Hkv, D, dtype=dtype)
    pos = torch.tensor([1, 4, 7], dtype=torch.int32, device="cuda")
    mask = z(N, B, dtype=torch.uint8)
    for kw in ({}, dict(scale=0.5, splits=3), dict(causal_block=True, ext_k=ek, ext_v=ev, E=4), dict(q_positions=pos, scaffold_mask=mask), dict(scale=2)):
        same(monkeypatch, M, lambda: Bd.fdd_block_attn_quant(q, p, L, bk, bv, out=out, workspace=ws, **kw))
    same(monkeypatch, M, lambda: Bd.fdd_block_attn_quant(q, p, 0, bk, bv, out=out, workspace=ws))


def test_log_probabilities(monkeypatch, M):
    N, B, V = 2, 5, 33
    for dtype in (torch.bfloat16, torch.float32):
        x, tok, mask = z(N, B, V, dtype=dtype), z(N, B, dtype=torch.int32), z(N, B, dtype=torch.uint8)
        for top, m in ((0, None), (4, mask)):
            outs = dict(logprobs=z(N, B, dtype=torch.float32), entropy=z(N, B, dtype=torch.float32), top_ids=z(N, B, top, dtype=torch.int32),
                        top_logprobs=z(N, B, top, dtype=torch.float32))
            same(monkeypatch, M, lambda: Bd.fdd_token_logprobs(x, tok, mask=m, top=top, temperature=0.7, **outs))
            same(monkeypatch, M, lambda: Bd.fdd_token_logprobs(x, tok, mask=m, top=top, temperature=1, **outs))


def test_wrong_arguments_are_left_to_python(M):
    p = Bd.fdd_quant_prefix(128, 2, 64)
    k = z(4, 2, 64)
    c = Bd.QuantCall()
    ok = lambda *a: M.quant(C.addressof(c), *a)
    assert ok(k, k, p, 0, 0)
    for bad in ((k.cpu(), k, p, 0, 0), (k, k.float(), p, 0, 0), (k, k[:2], p, 0, 0), (k, k, p[:3], 0, 0), (k, k, p, 125, 0), (k, k, p, -1, 0), (k, k, p, 0, 1),
                (k, k, p, 0, -1), (k.half(), k.half(), p, 0, 0), (k, k, p._replace(k_scale=p.k_scale.double()), 0, 0),
                (k, k, p._replace(v=p.v.view(torch.uint8)), 0, 0), (k, k, p._replace(v_scale=p.v_scale[:1]), 0, 0), (k, k, p, 0.0, 0)):
        assert not ok(*bad), bad
    with pytest.raises(ValueError, match="fit"):
        Bd.fdd_prefix_quantize(k, k, p, row0=125)
    with pytest.raises(TypeError, match="one element type"):
        Bd.fdd_prefix_quantize(k, k.float(), p)
    with pytest.raises(ValueError, match="GPU memory"):
        Bd.fdd_prefix_quantize(k.cpu(), k, p)
    q, b = z(1, 4, 4, 64), z(1, 4, 2, 64)
    with pytest.raises(ValueError, match="outside the cache"):
        Bd.fdd_block_attn_quant(q, p, 129, b, b)
    with pytest.raises(ValueError, match="Hkv and D"):
        Bd.fdd_block_attn_quant(z(1, 4, 4, 128), p, 1, z(1, 4, 2, 128), z(1, 4, 2, 128))
    with pytest.raises(TypeError, match="one element type"):
        Bd.fdd_block_attn_quant(q, p, 1, b.float(), b.float())
