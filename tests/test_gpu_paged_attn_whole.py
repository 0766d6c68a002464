"""Attention over a paged cache where a piece has many whole tiles: the steps that request nothing else, with four and eight wavefronts,
and prompts.  A tile that is lost or counted twice shows: every row's weight lies on two keys of its own, in tiles that follow one another."""
import numpy as np
import pytest
import torch

import paper_2605_23163_amd as F
from tests import paged_cut as cut
from tests.gpu_util import ROW_TOL
from tests.test_gpu_paged_attn import Call

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pointed:
    """Requests whose rows look at two keys each.  Keys have one length, so that both weigh about the same; K and V behind the last row are NaN."""

    def __init__(self, dtype, lens, B, Hq, Hkv, D, page, tile, seed):
        N, G, dt = len(lens), Hq // Hkv, DT[dtype]
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = np.random.default_rng(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
        even = lambda x: (x * (D ** 0.5 / x.norm(dim=-1, keepdim=True))).to(dt)
        need = [-(-L // page) for L in lens]
        pool = sum(need) + 2
        order = torch.randperm(pool, generator=g, device="cuda")
        table = torch.zeros(N, max(need) + 1, dtype=torch.int32, device="cuda")
        pages = [torch.full((pool, Hkv, page, D), float("nan"), dtype=dt, device="cuda") for _ in range(2)]
        self.q = torch.empty(N, B, Hq, D, dtype=dt, device="cuda")
        self.k, self.v = even(normal(N, B, Hkv, D)), normal(N, B, Hkv, D).to(dt)
        self.want = torch.empty(N, B, Hq, D, dtype=torch.float64, device="cuda")
        at = 0
        for n, L in enumerate(lens):
            mine = order[at:at + need[n]]
            table[n, :need[n]] = mine.int()
            at += need[n]
            kv = [even(normal(Hkv, L, D)), normal(Hkv, L, D).to(dt)]
            for p, x in zip(pages, kv):
                full = torch.full((Hkv, need[n] * page, D), float("nan"), dtype=dt, device="cuda")
                full[:, :L] = x
                p[mine] = full.view(Hkv, need[n], page, D).transpose(0, 1)
            starts = [(t * tile, min(tile, L - t * tile)) for t in range(-(-L // tile))] + [(L + t * tile, min(tile, B - t * tile)) for t in range(-(-B // tile))]
            for h in range(Hkv):
                k = torch.cat([kv[0][h], self.k[n, :, h]]).double()
                v = torch.cat([kv[1][h], self.v[n, :, h]]).double()
                rows = torch.arange(2 * B * G).numpy() + h      # two tiles a row, in order
                keys = [starts[t % len(starts)][0] + int(r.integers(0, starts[t % len(starts)][1])) for t in rows]
                q = (k[keys[::2]] + k[keys[1::2]]) * 4.0
                self.q[n, :, h * G:(h + 1) * G] = q.view(B, G, D).to(dt)
                q = self.q[n, :, h * G:(h + 1) * G].reshape(B * G, D).double()
                p = torch.softmax(q @ k.T.contiguous() * D ** -0.5, -1)
                self.want[n, :, h * G:(h + 1) * G] = (p @ v).view(B, G, D)
        self.cache = F.PagedCache(*pages, table, ints(lens))


# lens, B, Hq, Hkv, D, page; steps of whole tiles that some piece has in a row, at least
DEEP = [
    # eight wavefronts
    ([8192, 8000, 6001], 64, 28, 4, 128, 16, 4),
    ([16384], 64, 28, 4, 128, 64, 4),
    ([8192, 8192, 4099, 100, 5000, 8191, 7000, 8192], 64, 28, 4, 128, 128, 10),
    ([16384, 15001, 9999], 64, 28, 4, 64, 16, 8),
    ([4096] * 16, 32, 28, 4, 64, 32, 12),
    ([4096] * 16, 40, 28, 4, 128, 16, 20),
    # four
    ([4096] * 16, 8, 28, 4, 128, 16, 4),
    ([8000] * 14 + [3001, 8192], 4, 28, 4, 64, 64, 8),
    ([16384] * 12, 1, 28, 4, 128, 16, 16),
    ([5000] * 20, 16, 14, 2, 64, 16, 4),
]


@pytest.mark.parametrize("case", range(len(DEEP)))
def test_whole_tiles(case):
    """An output row's error: probabilities are rounded to 2^-8 of themselves, in the sum of their values and in their own, an average in fp16 to 2^-11 and
    the result to 2^-8, 1.2e-2 in all at worst.  A tile too few takes one of a row's two values away, one counted twice moves it by a third."""
    lens, B, Hq, Hkv, D, page, steps = DEEP[case]
    capacity = (max(-(-L // page) for L in lens) + 1) * page
    items = cut.items(lens, [B] * len(lens), B, Hq, Hkv, True, capacity)
    waves = cut.plan(len(lens), B, Hq, Hkv, True, capacity)[0]
    assert waves == (8 if case < 6 else 4) and max(i.whole for i in items) >= steps
    x = Pointed("bf16", lens, B, Hq, Hkv, D, page, 64, case)
    out = F.fdd_paged_attn(x.q, x.cache, x.k, x.v)
    err = ((out.double() - x.want).norm(dim=-1) / x.want.norm(dim=-1)).max().item()
    assert err <= ROW_TOL, err
    for _ in range(3):
        assert torch.equal(F.fdd_paged_attn(x.q, x.cache, x.k, x.v), out)


def test_the_check_sees_a_tile():
    """What a tile left out, or counted twice, does to the rows of a call like those above."""
    x = Pointed("bf16", [4096], 64, 7, 1, 128, 64, 64, 1)
    table = x.cache.page_table
    short = x.cache._replace(page_table=torch.cat([table[:, :20], table[:, 21:]], 1).contiguous(), lens=ints([4032]))
    double = x.cache._replace(page_table=torch.cat([table[:, :20], table[:, 19:-1]], 1).contiguous(), lens=ints([4160]))
    for cache in (short, double):
        out = F.fdd_paged_attn(x.q, cache, x.k, x.v)
        err = (out.double() - x.want).norm(dim=-1) / x.want.norm(dim=-1)
        assert (err > 4 * ROW_TOL).sum() >= 7        # (448 rows of two keys each look at 65 tiles: 13 or more at each)


@pytest.mark.parametrize("lens,B,tile", [([2048, 1777], 16, 32), ([6000], 3, 32)])
def test_whole_tiles_in_fp32(lens, B, tile):
    """fp32 products and sums: scores up to 2^6 of 128 products are off by 2^-11 of 1 at most (130 roundings of 2^-24 of them), and a weight by that."""
    x = Pointed("f32", lens, B, 28, 4, 128, 16, tile, 7)
    out = F.fdd_paged_attn(x.q, x.cache, x.k, x.v)
    err = ((out.double() - x.want).norm(dim=-1) / x.want.norm(dim=-1)).max().item()
    assert err <= 2.0 ** -9, err


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,B,Hq,Hkv,D,page,counts,mode", [
    ([0], 1100, 7, 1, 128, 16, None, "causal"), ([0, 0, 5], 500, 14, 2, 64, 16, [500, 333, 1], "causal"), ([700, 33], 600, 14, 2, 128, 64, [600, 433], "causal"),
    ([2500], 513, 4, 1, 64, 256, None, "causal"), ([0], 700, 7, 1, 128, 16, None, "full"), ([90], 450, 7, 1, 64, 32, None, "any")])
def test_prompts(dtype, lens, B, Hq, Hkv, D, page, counts, mode):
    """Hundreds of tokens in one call: M-tiles that see few of the request's own tiles beside some that see all."""
    x = Call(dtype, lens, B, Hq, Hkv, D, page, counts, mode, seed=B)
    x.check(x.run())
