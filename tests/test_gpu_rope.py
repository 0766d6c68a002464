"""Rotary positions on the GPU against 64 bits, and their gradient."""
import numpy as np
import pytest
import torch

import paper_2605_23163_amd as F
from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def check(got, x, positions, w, m, interleaved, bf16, inverse=False):
    x = x.double().cpu().numpy()
    want = R.rotate(x, positions.cpu().numpy(), w, m, interleaved, inverse)
    bound = R.rotate_bound(x, w, m, interleaved, bf16, want)
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= bound), f"{(err - bound).max()} above the bound"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lead,Hq,Hk,D,R_,interleaved,scaling", [
    ((1,), 1, 1, 64, 64, False, None), ((3, 5), 28, 4, 128, 128, False, None), ((3, 5), 28, 4, 128, 128, True, "linear"), ((7,), 4, 1, 64, 32, False, "base"),
    ((7,), 4, 1, 64, 32, True, "parts"), ((2, 3), 3, 2, 128, 24, False, None), ((2, 3), 3, 2, 128, 24, True, None), ((5,), 2, 3, 7, 6, False, None), ((5,), 2, 3, 10, 2, True, None),
    ((300, 9), 14, 2, 64, 64, False, "parts"), ((1000,), 8, 8, 256, 128, True, None), ((3,), 1, 0, 1024, 1024, False, None)])
def test_rope(dtype, lead, Hq, Hk, D, R_, interleaved, scaling):
    g = torch.Generator(device="cuda").manual_seed(5)
    how = dict(scaling=scaling, stretch=4.0, original=4096) if scaling else {}
    table = F.fdd_rope_table(R_, base=1e4, interleaved=interleaved, **how)
    w, m = R.frequencies(R_, 1e4, scaling, 4.0, 4096)
    q = torch.randn(lead + (Hq, D), generator=g, device="cuda").to(DT[dtype])
    k = torch.randn(lead + (Hk, D), generator=g, device="cuda").to(DT[dtype]) if Hk else None
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, lead, generator=g, device="cuda").to(torch.int32)
    pos.view(-1)[0] = (1 << 31) - 1
    before = q.clone()
    out = F.fdd_rope(q, pos, table, k=k)
    for o, x in ([(out, q)] if k is None else list(zip(out, (q, k)))):
        check(o, x, pos, w, m, interleaved, dtype == "bf16")
        assert torch.equal(o[..., R_:], x[..., R_:])
    assert torch.equal(before, q)
    # in place, on another stream, and back again
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    x = q.clone()
    s.wait_stream(torch.cuda.current_stream())
    y = F.fdd_rope(x, pos, table, out=x, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert y is x and torch.equal(x, out if k is None else out[0])
    check(F.fdd_rope(x, pos, table, inverse=True), x, pos, w, m, interleaved, dtype == "bf16", inverse=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_rope_of_parts_of_a_projection(dtype, offset):
    """q and k lie in wider rows, at any alignment of the type; in place."""
    N, B, Hq, Hk, D = 2, 3, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(6)
    table = F.fdd_rope_table(D)
    w, m = R.frequencies(D, 1e4)
    wide = torch.randn(N * B * ((Hq + 2 * Hk) * D + 2 * offset) + offset, generator=g, device="cuda").to(DT[dtype])
    rows = wide[offset:].view(N, B, -1)
    q = rows[..., :Hq * D].unflatten(2, (Hq, D))
    k = rows[..., Hq * D:(Hq + Hk) * D].unflatten(2, (Hk, D))
    rest = rows[..., (Hq + Hk) * D:].clone()
    pos = torch.arange(N * B, dtype=torch.int32, device="cuda").view(N, B) + 100000
    q0, k0 = q.clone(), k.clone()
    F.fdd_rope(q, pos, table, k=k, out=q, k_out=k)
    check(q, q0, pos, w, m, False, dtype == "bf16")
    check(k, k0, pos, w, m, False, dtype == "bf16")
    assert torch.equal(rows[..., (Hq + Hk) * D:], rest)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_gradient(interleaved):
    """The rotation is linear: <rope(x + d) - rope(x), g> is <d, inverse(g)>, by formula and by differences."""
    table = F.fdd_rope_table(48, interleaved=interleaved, scaling="parts", stretch=8.0, original=2048)
    g0 = torch.Generator(device="cuda").manual_seed(7)
    x, d, g = (torch.randn(5, 3, 64, generator=g0, device="cuda") for _ in range(3))
    pos = torch.tensor([0, 1, 4096, 99999, -5], dtype=torch.int32, device="cuda")
    grad = F.fdd_rope(g, pos, table, inverse=True)
    w, m = R.frequencies(48, 1e4, "parts", 8.0, 2048)
    check(grad, g, pos, w, m, interleaved, False, inverse=True)
    left = ((F.fdd_rope(x + d, pos, table) - F.fdd_rope(x, pos, table)).double() * g.double()).sum()
    right = (d.double() * grad.double()).sum()
    # each of 2 * 960 rotated values is off by 2^-21 (|u| + |v|) m at most, and the sum x + d by half a step
    assert abs(float(left - right)) <= 3 * 960 * 2.0 ** -21 * 10 * m * 5


def test_rope_in_a_graph_follows_its_positions():
    table = F.fdd_rope_table(128)
    x = torch.randn(4, 2, 128, device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    F.fdd_rope(x, pos, table, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        F.fdd_rope(x, pos, table, out=out)
    for p in (3, 70000, 5):
        pos.fill_(p)
        graph.replay()
        eager = F.fdd_rope(x, pos, table)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_rope_of_nothing_and_of_wrong_arguments():
    table = F.fdd_rope_table(64)
    e = F.fdd_rope(torch.empty(0, 2, 64, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), table)
    assert e.shape == (0, 2, 64)
    x, pos = torch.randn(4, 2, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        F.fdd_rope(x.transpose(1, 2), pos, table)
    with pytest.raises(ValueError):
        F.fdd_rope(x[:1].expand(4, 2, 64), pos, table)
    with pytest.raises(ValueError):
        F.fdd_rope(x, pos, table, out=torch.empty(4, 3, 64, device="cuda"))
    with pytest.raises(TypeError):
        F.fdd_rope(x, pos, table, k=x.bfloat16())
    with pytest.raises(F.FddError):
        F.fdd_rope(x[:3], pos[:3], table, out=x[1:])
    with pytest.raises(F.FddError):
        F.fdd_rope(x[..., :32].contiguous(), pos, table)


@pytest.mark.parametrize("dtype,rows,Hq,D,interleaved", [("bf16", 1100, 128, 128, False), ("f32", 1100, 64, 128, True)])
def test_rope_of_many_rows(dtype, rows, Hq, D, interleaved):
    """More than the caches hold: 36 MB written."""
    g = torch.Generator(device="cuda").manual_seed(9)
    table = F.fdd_rope_table(D, interleaved=interleaved)
    q = torch.randn(rows, Hq, D, generator=g, device="cuda").to(DT[dtype])
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") * 17 + 5
    w, m = R.frequencies(D, 1e4)
    check(F.fdd_rope(q, pos, table), q, pos, w, m, interleaved, dtype == "bf16")
