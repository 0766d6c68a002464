"""The 8-bit prefix cache and token log probabilities on a machine without a GPU: every mistake that the host can see is a
status code or an exception and nothing is launched; and the reference in 64 bits against cases worked out by hand."""
import ctypes as C
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2605_23163_amd import binding as bd
from tests import quant_ref as Q


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(bd.library_path()):
        from paper_2605_23163_amd import build
        build.build()
    return bd.load_library()


def fill(p, base, kw):
    for k, v in {**base, **kw}.items():
        setattr(p, k, v)
    return p


def cache(**kw):
    return fill(bd.QuantCache(), dict(k=1 << 20, v=1 << 21, k_scale=1 << 22, v_scale=1 << 23, Hkv=4, D=128, capacity=256), kw)


def rows(**kw):
    return fill(bd.QuantRows(), dict(k=1 << 24, v=1 << 25, rows=32, dtype=bd.FDD_BF16), kw)


def attn(**kw):
    return fill(bd.AttnParams(), dict(N=1, B=32, L=200, Hq=28, Hkv=4, D=128, dtype=bd.FDD_BF16, q=256, block_k=1024, block_v=1280, out=1536,
                                      workspace=1 << 30, workspace_bytes=1 << 30), kw)


def logp(**kw):
    return fill(bd.LogprobParams(), dict(N=2, B=8, V=1000, dtype=bd.FDD_BF16, top=4, temperature=1.0, logits=256, tokens=512, logprobs=768,
                                         entropy=1024, top_ids=1280, top_logprobs=1536, workspace=1 << 30, workspace_bytes=1 << 30), kw)


@pytest.mark.parametrize("fn", ["fdd_prefix_quantize", "fdd_prefix_dequantize"])
def test_rows_are_checked(lib, fn):
    f = getattr(lib, fn)
    for ckw, rkw, row0, code in [
            (dict(Hkv=0), {}, 0, 2), (dict(capacity=100), {}, 0, 2), (dict(capacity=0), {}, 0, 2), (dict(D=96), {}, 0, 4), (dict(reserved=1), {}, 0, 4),
            (dict(capacity=1 << 30), {}, 0, 2), (dict(k=None), {}, 0, 1), (dict(v_scale=None), {}, 0, 1), (dict(v=8), {}, 0, 4), (dict(k_scale=2), {}, 0, 4),
            ({}, {}, -1, 2), ({}, {}, 225, 2), ({}, dict(rows=-1), 0, 2), ({}, dict(rows=2 ** 31 - 1), 2 ** 31 - 1, 2), ({}, dict(dtype=2), 0, 3),
            ({}, dict(k=None), 0, 1), ({}, dict(v=8), 0, 4), ({}, dict(k_row_stride=511), 0, 2), ({}, dict(v_row_stride=516), 0, 2),
            ({}, dict(v_row_stride=-512), 0, 2), ({}, dict(k_row_stride=1 << 40), 0, 2),
            ({}, dict(k=1 << 20), 0, 4), ({}, dict(v=(1 << 21) + 4 * 256 * 128 - 16), 0, 4), ({}, dict(k=(1 << 22) - 1024), 0, 4)]:
        assert f(C.byref(cache(**ckw)), row0, C.byref(rows(**rkw)), None) == code, (ckw, rkw, row0)
        assert lib.fdd_last_error().decode().startswith(fn + ":")
    assert f(None, 0, C.byref(rows()), None) == 1
    assert f(C.byref(cache()), 0, None, None) == 1
    # nothing to move: no launch, no pointers needed
    assert f(C.byref(cache()), 256, C.byref(rows(rows=0, k=None, v=None)), None) == 0


def test_attention_is_checked(lib):
    f = lib.fdd_block_attn_quant
    for kw, ckw, code in [(dict(N=0), {}, 2), (dict(L=-1), {}, 2), (dict(Hq=30), {}, 2), (dict(dtype=2), {}, 3), (dict(D=96), {}, 4), (dict(flags=2), {}, 4),
                          (dict(splits=65), {}, 4), (dict(q=None), {}, 1), (dict(block_v=None), {}, 1), (dict(out=256), {}, 4), (dict(q=264), {}, 4),
                          (dict(scale=float("inf")), {}, 4), (dict(E=4, ext_capacity=4), {}, 1), (dict(n_q_positions=3), {}, 1), (dict(n_q_positions=33), {}, 2),
                          (dict(prefix_k=512), {}, 4), (dict(prefix_v_packed=512), {}, 4),
                          (dict(L=257), {}, 2), ({}, dict(Hkv=2), 2), ({}, dict(D=64), 2), ({}, dict(capacity=100), 2), ({}, dict(k=None), 1), ({}, dict(v=4), 4),
                          (dict(batch=2, q_batch_stride=1 << 20, out_batch_stride=1 << 20, block_batch_stride=1 << 20), {}, 2),
                          (dict(batch=2, q_batch_stride=1 << 20, out_batch_stride=1 << 20, block_batch_stride=1 << 20),
                           dict(batch_stride=4 * 256 * 128 + 8, scale_batch_stride=16), 2),
                          (dict(batch=2, q_batch_stride=1 << 20, out_batch_stride=1 << 20, block_batch_stride=1 << 20),
                           dict(batch_stride=4 * 256 * 128, scale_batch_stride=15), 2),
                          (dict(batch=2, q_batch_stride=100, out_batch_stride=1 << 20, block_batch_stride=1 << 20), {}, 2)]:
        assert f(C.byref(attn(**kw)), C.byref(cache(**ckw))) == code, (kw, ckw)
        assert lib.fdd_last_error().decode().startswith("fdd_block_attn_quant:"), (kw, ckw)
    assert f(None, C.byref(cache())) == 1
    assert f(C.byref(attn()), None) == 1
    need = lib.fdd_block_attn_quant_workspace(C.byref(attn(L=4096)))
    assert need > 0 and need % 256 == 0
    for kw in (dict(workspace=None), dict(workspace=(1 << 30) + 4), dict(workspace_bytes=need - 1)):
        assert f(C.byref(attn(L=4096, **kw)), C.byref(cache(capacity=4096))) == 5, kw
    assert lib.fdd_block_attn_quant_workspace(C.byref(attn(Hq=30))) == 0


def test_logprobs_are_checked(lib):
    f = lib.fdd_token_logprobs
    for kw, code in [(dict(N=0), 2), (dict(B=-1), 2), (dict(V=0), 2), (dict(V=1 << 31), 2), (dict(N=1 << 20, B=1 << 10), 2), (dict(dtype=2), 3),
                     (dict(top=-1), 2), (dict(top=33), 2), (dict(V=3), 2), (dict(temperature=0.0), 4), (dict(temperature=-1.0), 4),
                     (dict(temperature=float("nan")), 4), (dict(temperature=float("inf")), 4), (dict(temperature=1e-45), 4), (dict(reserved=1), 4),
                     (dict(logits=None), 1), (dict(tokens=None), 1), (dict(top_ids=None), 1), (dict(top_logprobs=None), 1), (dict(logits=264), 4),
                     (dict(entropy=1026), 4), (dict(logprobs=None, entropy=None, top=0), 1)]:
        assert f(C.byref(logp(**kw))) == code, kw
        assert lib.fdd_last_error().decode().startswith("fdd_token_logprobs:")
    assert f(None) == 1
    need = lib.fdd_token_logprobs_workspace(C.byref(logp(V=152064, top=20)))
    if need:
        for kw in (dict(workspace=None), dict(workspace=(1 << 30) + 4), dict(workspace_bytes=need - 1)):
            assert f(C.byref(logp(V=152064, top=20, **kw))) == 5, kw
    assert lib.fdd_token_logprobs_workspace(C.byref(logp(V=0))) == 0


def test_smallest_temperature(lib):
    """1 / 4e-39 is an fp32 number, log2(e) / 4e-39 is none."""
    assert lib.fdd_token_logprobs(C.byref(logp(temperature=4e-39))) == 4
    assert "temperature" in lib.fdd_last_error().decode()


def host_prefix(cap=128, Hkv=2, D=64, **kw):
    d = dict(k=torch.zeros(Hkv, cap, D).to(torch.float8_e4m3fn), v=torch.zeros(Hkv, cap, D).to(torch.float8_e4m3fn),
             k_scale=torch.ones(Hkv, cap // 64), v_scale=torch.ones(Hkv, cap // 64))
    d.update(kw)
    return bd.QuantPrefix(**d)


def test_binding_refuses(lib):
    bf = torch.bfloat16
    x = torch.zeros(3, 2, 64, dtype=bf)
    good = host_prefix()
    with pytest.raises(ValueError, match="GPU memory"):
        bd.fdd_prefix_quantize(x, x, good)
    with pytest.raises(ValueError, match="capacity"):
        bd.fdd_prefix_quantize(x, x, host_prefix(v_scale=torch.ones(2, 3)))
    with pytest.raises(TypeError, match="float8"):
        bd.fdd_prefix_quantize(x, x, host_prefix(k=torch.zeros(2, 128, 64, dtype=torch.int8)))
    q, b = torch.zeros(1, 4, 4, 64, dtype=bf), torch.zeros(1, 4, 2, 64, dtype=bf)
    with pytest.raises(ValueError, match="outside the cache"):
        bd.fdd_block_attn_quant(q, None, 1, b, b)
    with pytest.raises(ValueError, match="GPU memory"):
        bd.fdd_block_attn_quant(q, None, 0, b, b)
    with pytest.raises(ValueError, match="leading dimension"):
        bd.fdd_block_attn_quant_batched(q[None], good, 1, b[None], b[None])
    logits, tok = torch.zeros(1, 2, 50), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(TypeError, match="tokens"):
        bd.fdd_token_logprobs(logits, tok.long())
    with pytest.raises(TypeError, match="mask"):
        bd.fdd_token_logprobs(logits, tok, mask=torch.ones(1, 2, dtype=torch.bool))
    with pytest.raises(ValueError, match="top"):
        bd.fdd_token_logprobs(logits, tok, top=33)
    with pytest.raises(TypeError, match="entropy"):
        bd.fdd_token_logprobs(logits, tok, entropy=torch.zeros(2, 1))
    with pytest.raises(TypeError, match="top_ids"):
        bd.fdd_token_logprobs(logits, tok, top=2, top_ids=torch.zeros(1, 2, 3, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU memory"):
        bd.fdd_token_logprobs(logits, tok)


FIRST_CALLS = {
    "fdd_block_attn_quant_workspace": "F.fdd_block_attn_quant_workspace(q, p, 1, b, b)",
    "fdd_block_attn_quant_batched_workspace": "F.fdd_block_attn_quant_batched_workspace(q[None], P, 1, b[None], b[None])",
    "fdd_token_logprobs_workspace": "F.fdd_token_logprobs_workspace(b.float()[0])",
    "fdd_block_attn_quant": "F.fdd_block_attn_quant(q, p, 1, b, b)",
    "fdd_block_attn_quant_batched": "F.fdd_block_attn_quant_batched(q[None], P, 1, b[None], b[None])",
    "fdd_prefix_quantize": "F.fdd_prefix_quantize(b[0], b[0], p)",
    "fdd_prefix_dequantize": "F.fdd_prefix_dequantize(p, 4, k=b[0], v=b[0])",
    "fdd_token_logprobs": "F.fdd_token_logprobs(b.float()[0], torch.zeros(4, 2, dtype=torch.int32))",
    "fdd_quant_prefix": "F.fdd_quant_prefix(100, 2, 64, device='cpu')",
}


@pytest.mark.parametrize("name", sorted(FIRST_CALLS))
def test_any_call_may_be_the_first(name):
    """The library and torch are loaded by the first call, whichever it is; host tensors are refused as such."""
    code = f"""
import torch
import paper_2605_23163_amd as F
q, b = torch.zeros(1, 4, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
p = F.QuantPrefix(*(torch.zeros(2, 64, 64).to(torch.float8_e4m3fn) for _ in range(2)), *(torch.ones(2, 1) for _ in range(2)))
P = F.QuantPrefix(*(t[None] for t in p))
try:
    {FIRST_CALLS[name]}
    print("returned")
except ValueError as e:
    print("refused", "GPU memory" in str(e))
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert r.stdout.strip() in (("returned",) if name in ("fdd_quant_prefix", "fdd_token_logprobs_workspace") else ("refused True",)), r.stdout


class Elsewhere:
    """Stands in for a tensor on another device than the current one."""
    is_cuda = True
    device = torch.device("cuda", 5)


def test_other_devices_are_refused(monkeypatch, lib):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        bd._on_current_device(None, Elsewhere())


def test_reference_by_hand():
    # 449 needs the next power of two, 448 does not; the least and the largest scale
    assert Q.scale_of(np.array([448.0, -3])) == 1.0 and Q.scale_of(np.array([-449.0])) == 2.0 and Q.scale_of(np.array([224.0])) == 0.5
    assert Q.scale_of(np.zeros(4)) == 2.0 ** -117 and Q.scale_of(np.array([np.inf, np.nan])) == 2.0 ** -117
    assert Q.scale_of(np.array([np.finfo(np.float32).max])) == 2.0 ** 119
    # ties go to the even code: 1 + 1/16 lies between 1 (0x38) and 1.125 (0x39), 1 + 3/16 between 0x39 and 0x3a
    assert list(Q.encode(np.array([1.0625, 1.1875, -1.0625, 0.0, -0.0, 1e9, -np.inf, 2.0 ** -10, 3 * 2.0 ** -10, np.nan]), 1.0)) == \
        [0x38, 0x3a, 0xb8, 0, 0x80, 0x7e, 0xfe, 0, 2, 0x7f]
    for c in range(256):
        if c & 127 != 127:
            assert Q.encode(Q.VALUES[c:c + 1], 1.0)[0] == c
            assert torch.tensor([c], dtype=torch.uint8).view(torch.float8_e4m3fn).float().item() == Q.VALUES[c]
