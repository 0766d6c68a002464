"""fdd_prefix_dequantize writes rows of K and rows of V: they may be parts of wider rows, but must not share bytes."""
import ctypes as C

import pytest
import torch

from paper_2605_23163_amd import binding as bd
from tests.test_quant_args import cache, lib, rows  # noqa: F401

K = 1 << 24
ROW = 4 * 128                 # elements of a row of the cache of test_quant_args


@pytest.mark.parametrize("dtype,es", [(bd.FDD_BF16, 2), (bd.FDD_F32, 4)])
def test_rows_that_share_bytes_are_refused(lib, dtype, es):  # noqa: F811
    row = ROW * es
    for v, n, sk, sv in [(K, 32, 0, 0), (K, 1, 0, 0), (K + row - 16, 1, 0, 0), (K - row + 16, 1, 0, 0), (K + 16, 32, 0, 0), (K + 31 * row, 32, 0, 0),
                         (K - 31 * row, 32, 0, 0), (K + row // 2, 32, 3 * ROW, 3 * ROW), (K + 3 * row - 16, 32, 3 * ROW, 3 * ROW),
                         (K - 3 * row + 16, 32, 3 * ROW, 3 * ROW), (K + 3 * 31 * row + row - 16, 32, 3 * ROW, 3 * ROW),
                         (K + row, 32, 3 * ROW, 4 * ROW),                 # row 2 of V is row 3 of K
                         (K + 2 * row, 32, 3 * ROW, 0), (K - 2 * row, 32, 0, 5 * ROW), (K + 31 * 3 * row, 32, 3 * ROW, 7 * ROW), (K - 31 * 7 * row, 32, 3 * ROW, 7 * ROW)]:
        r = rows(k=K, v=v, rows=n, k_row_stride=sk, v_row_stride=sv, dtype=dtype)
        assert lib.fdd_prefix_dequantize(C.byref(cache()), 0, C.byref(r), None) == 4, (v - K, n, sk, sv)
        assert "overlap" in lib.fdd_last_error().decode()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_may_interleave(dtype):
    import paper_2605_23163_amd as F
    Hkv, D, n = 2, 64, 70
    w = Hkv * D
    x = torch.randn(n, Hkv, D, device="cuda", dtype=dtype)
    p = F.fdd_quant_prefix(n, Hkv, D)
    F.fdd_prefix_quantize(x, -x, p)
    ref = F.fdd_prefix_dequantize(p, n, dtype=dtype)
    part = lambda buf, at, stride, m: buf.as_strided((m, Hkv, D), (stride, D, 1), at)
    # (start and stride of k, of v, rows): parts of one row either way round, rows apart, rows of different strides that pass one another
    for ka, ks, va, vs, m in [(0, 2 * w, w, 2 * w, n), (w, 2 * w, 0, 2 * w, n), (0, 3 * w, 5 * w, 3 * w, n), (7 * w, 3 * w, 0, 3 * w, n), (0, w, n * w, w, n),
                              (n * w, w, 0, w, n), (0, 4 * w, w, 6 * w, n), (0, 2 * w, 3 * w, 4 * w, n), (0, 0, w, 0, 1)]:
        buf = torch.full((800 * w,), 7.0, dtype=dtype, device="cuda")
        k, v = part(buf, ka, ks, m), part(buf, va, vs, m)
        F.fdd_prefix_dequantize(p, m, k=k, v=v)
        assert torch.equal(k, ref[0][:m]) and torch.equal(v, ref[1][:m]), (ka, ks, va, vs)
        assert int((buf != 7.0).sum()) <= 2 * m * w
    with pytest.raises(F.FddError, match="overlap"):
        F.fdd_prefix_dequantize(p, n, k=x, v=x)


def test_a_cache_whose_arrays_overlap_is_not_written(lib):  # noqa: F811
    codes, scales = 4 * 256 * 128, 4 * 4 * 4
    for kw in (dict(v=1 << 20), dict(v=(1 << 20) + codes - 16), dict(v=(1 << 20) - codes + 16), dict(v_scale=1 << 22), dict(v_scale=(1 << 22) + scales - 4),
               dict(k_scale=1 << 20), dict(k_scale=(1 << 21) + codes - 4), dict(v_scale=(1 << 20) - scales + 4), dict(v_scale=1 << 21)):
        assert lib.fdd_prefix_quantize(C.byref(cache(**kw)), 0, C.byref(rows()), None) == 4, kw
        assert "overlap" in lib.fdd_last_error().decode()
