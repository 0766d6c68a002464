"""The caller's output of attention over the 8-bit cache has to be what the library writes: as many elements as q, of its type.

Nothing is launched here: the binding refuses host tensors after it has looked at shapes and types, and the native marshalling only
fills a struct."""
import ctypes as C
import os

import pytest
import torch

from paper_2605_23163_amd import binding as bd
from tests.test_quant_args import host_prefix

BF = torch.bfloat16
WRONG = [((1, 4, 4, 64), torch.float32), ((1, 3, 4, 64), BF), ((2, 4, 4, 64), BF), ((4, 4, 64), BF), ((1, 4, 2, 64), BF), ((16, 64), BF), ((0,), BF)]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(bd.library_path()):
        from paper_2605_23163_amd import build
        build.build()
    return bd.load_library()


@pytest.mark.parametrize("shape,dtype", WRONG)
def test_out_is_checked(lib, shape, dtype):
    q, b = torch.zeros(1, 4, 4, 64, dtype=BF), torch.zeros(1, 4, 2, 64, dtype=BF)
    out = torch.zeros(shape, dtype=dtype)
    for prefix in (host_prefix(), None):
        with pytest.raises((ValueError, TypeError), match="out must have"):
            bd.fdd_block_attn_quant(q, prefix, 0 if prefix is None else 5, b, b, out=out)
        with pytest.raises((ValueError, TypeError), match="out must have"):
            bd.fdd_block_attn_quant(q, prefix, 0 if prefix is None else 5, b, b, out=out, q_positions=torch.zeros(3, dtype=torch.int32))
    batch = bd.QuantPrefix(*(t.expand(2, *t.shape) for t in host_prefix()))
    two = lambda t: t.expand(2, *t.shape).contiguous()
    with pytest.raises((ValueError, TypeError), match="out must have"):
        bd.fdd_block_attn_quant_batched(two(q), batch, 5, two(b), two(b), out=two(out))
    with pytest.raises((ValueError, TypeError), match="out must have"):
        bd.fdd_block_attn_quant_batched(two(q), batch, 5, two(b), two(b), out=two(q)[:1])


def test_right_out_passes_these_checks(lib):
    q, b = torch.zeros(1, 4, 4, 64, dtype=BF), torch.zeros(1, 4, 2, 64, dtype=BF)
    with pytest.raises(ValueError, match="GPU memory"):
        bd.fdd_block_attn_quant(q, host_prefix(), 5, b, b, out=torch.empty_like(q))


@pytest.mark.gpu
@pytest.mark.parametrize("shape,dtype", WRONG)
def test_marshalling_leaves_a_wrong_out_to_python(lib, shape, dtype):
    if bd._marshal is None:
        pytest.skip("built without torch's headers")
    z = lambda *s, dtype=BF: torch.zeros(s, dtype=dtype, device="cuda")
    q, b, p, c = z(1, 4, 4, 64), z(1, 4, 2, 64), bd.fdd_quant_prefix(64, 2, 64), bd.AttnQuantCall()
    fill = lambda out: bd._marshal.attn_quant(C.addressof(c), q, p, 5, b, b, None, out, None, None, None, 0, False, 0, None, torch.cuda.current_device())
    assert fill(torch.empty_like(q))
    assert not fill(z(*shape, dtype=dtype))
