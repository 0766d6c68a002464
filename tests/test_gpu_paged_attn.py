"""Attention over a paged cache on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_23163_amd as F
from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Call:
    """A call's inputs.  What must not be used is filled with NaN: rows behind the last one of a page, pages that nobody lists, tokens
    that are not there."""

    def __init__(self, dtype, lens, B, Hq, Hkv, D, page, counts=None, mode="full", seed=0, spread=1.0, extra_pages=1, strided=False):
        N = len(lens)
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = np.random.default_rng(seed)
        self.N, self.B, self.Hq, self.Hkv, self.D, self.page, self.lens, self.mode = N, B, Hq, Hkv, D, page, list(lens), mode
        self.dtype, self.bf16 = DT[dtype], dtype == "bf16"
        self.counts = [B] * N if counts is None else list(counts)
        t = self.dtype
        need = [(n + page - 1) // page for n in lens]
        pool = sum(need) + 3
        order = torch.randperm(pool, generator=g, device="cuda").tolist()
        wide = max(need) + extra_pages
        table = np.full((N, wide), -7, dtype=np.int64)
        table[:, -1] = 1 << 30
        at = 0
        for n in range(N):
            table[n, :need[n]] = order[at:at + need[n]]
            at += need[n]
        kv = []
        for _ in range(2):
            p = torch.full((pool, Hkv, page, D), float("nan"), dtype=t, device="cuda")
            for n in range(N):
                for i in range(need[n]):
                    rows = min(page, lens[n] - i * page)
                    p[table[n, i], :, :rows] = (torch.randn(Hkv, rows, D, generator=g, device="cuda") * spread).to(t)
            kv.append(p)
        self.cache = F.PagedCache(*kv, ints(table.tolist()), ints(self.lens))
        if strided:
            fused = (torch.randn(N, B, (Hq + 2 * Hkv) * D, generator=g, device="cuda") * spread).to(t)
            self.q = fused[..., :Hq * D].unflatten(2, (Hq, D))
            self.k = fused[..., Hq * D:(Hq + Hkv) * D].unflatten(2, (Hkv, D))
            self.v = fused[..., (Hq + Hkv) * D:].unflatten(2, (Hkv, D))
        else:
            self.q, self.k, self.v = ((torch.randn(N, B, h, D, generator=g, device="cuda") * spread).to(t) for h in (Hq, Hkv, Hkv))
        for n in range(N):
            for x in (self.q, self.k, self.v):
                x[n, self.counts[n]:] = float("nan")
        self.see = []
        for n in range(N):
            c = self.counts[n]
            if mode == "full":
                self.see.append(np.ones((c, c), dtype=bool))
            elif mode == "causal":
                self.see.append(np.tril(np.ones((c, c), dtype=bool)))
            elif mode == "tree":
                self.see.append(R.ancestors([-1] + [int(r.integers(max(0, i - 4), i)) for i in range(1, B)], c))
            else:                                   # any pattern, rows that see nothing among them
                m = r.random((c, c)) < 0.4
                m[::3] = False
                self.see.append(m)
        self.mask = None
        if mode in ("tree", "any"):
            words = np.zeros((N, B, (B + 63) // 64), dtype=np.int64)
            words[:] = -1                            # bits of tokens that are not there mean nothing
            for n in range(N):
                c = self.counts[n]
                bits = np.ones((c, (B + 63) // 64 * 64), dtype=bool)
                bits[:, :c] = self.see[n]
                words[n, :c] = np.packbits(bits, axis=1, bitorder="little").view(np.int64)
            self.mask = torch.from_numpy(words).cuda()

    def run(self, **kw):
        if "n_tokens" not in kw:
            kw["n_tokens"] = ints(self.counts)
        return F.fdd_paged_attn(self.q, self.cache, self.k, self.v, mask=self.mask, causal_block=self.mode == "causal", **kw)

    def check(self, out, scale=None, max_len=None, untouched=0.0):
        D, G, page = self.D, self.Hq // self.Hkv, self.page
        scale = D ** -0.5 if scale is None else scale
        f = lambda t: t.double().cpu().numpy()
        kp, vp, q, k, v, o = (f(t) for t in (self.cache.k, self.cache.v, self.q, self.k, self.v, out))
        table = self.cache.page_table.cpu().numpy()
        for n in range(self.N):
            L, c = self.lens[n] if max_len is None else min(self.lens[n], max_len), self.counts[n]
            assert np.all(o[n, c:] == untouched), "rows of tokens that are not there were written"
            if c == 0:
                continue
            pages = table[n, :(L + page - 1) // page]
            for h in range(self.Hkv):
                kk = np.concatenate([kp[pages, h].reshape(-1, D)[:L], k[n, :c, h]])
                vv = np.concatenate([vp[pages, h].reshape(-1, D)[:L], v[n, :c, h]])
                qq = q[n, :c, h * G:(h + 1) * G].reshape(c * G, D)
                see = np.concatenate([np.ones((c * G, L), dtype=bool), np.repeat(self.see[n], G, 0)], 1)
                want, a = R.attention(qq, kk, vv, see, scale)
                bound = R.attention_bound(qq, kk, scale, want, a, self.bf16)
                err = np.abs(o[n, :c, h * G:(h + 1) * G].reshape(c * G, D) - want)
                assert np.all(err <= bound), f"request {n} head {h}: {np.nanmax(err - bound)} above the bound, {np.isnan(err).sum()} NaN"


SHAPES = [
    # lens, B, Hq, Hkv, D, page, counts, mode
    ([1], 1, 1, 1, 64, 16, None, "full"),
    ([0], 1, 4, 1, 128, 16, None, "causal"),
    ([0, 1, 15, 16, 17, 63, 64, 65], 1, 28, 4, 128, 16, None, "full"),
    ([500, 31, 2000], 1, 8, 8, 64, 32, None, "causal"),
    ([129, 0, 64], 5, 14, 2, 64, 16, [5, 0, 3], "tree"),
    ([300, 77], 16, 28, 4, 128, 64, [16, 9], "tree"),
    ([1000, 3], 32, 28, 4, 128, 128, [32, 17], "tree"),
    ([700, 4097], 37, 28, 4, 128, 64, [37, 30], "causal"),
    ([64, 640], 64, 28, 4, 128, 16, None, "full"),
    ([10, 333], 65, 4, 1, 64, 256, [65, 64], "tree"),
    ([200], 130, 8, 2, 128, 64, None, "causal"),
    ([63, 0], 200, 4, 2, 64, 32, [200, 129], "tree"),
    ([0, 0, 90], 12, 6, 2, 128, 16, [12, 1, 7], "any"),
    ([0, 5], 100, 3, 1, 64, 64, [100, 70], "any"),
    ([1024, 1023, 1025], 3, 32, 8, 128, 1024, None, "causal"),
    ([3000], 8, 7, 7, 64, 16, None, "tree"),
    ([2500, 100], 70, 16, 4, 128, 64, [70, 33], "full"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_attention(dtype, case):
    lens, B, Hq, Hkv, D, page, counts, mode = SHAPES[case]
    x = Call(dtype, lens, B, Hq, Hkv, D, page, counts, mode, seed=case, strided=case % 2 == 1)
    x.check(x.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seed", range(12))
def test_random_calls(dtype, seed):
    r = np.random.default_rng(100 + seed)
    N, B = int(r.integers(1, 6)), int(r.choice([1, 2, 7, 16, 33, 64, 90]))
    Hkv = int(r.choice([1, 2, 4]))
    Hq = Hkv * int(r.choice([1, 2, 5, 7, 8]))
    lens = [int(np.exp(r.uniform(0, np.log(3000)))) - 1 for _ in range(N)]
    counts = [int(r.integers(0, B + 1)) for _ in range(N)]
    mode = ["full", "causal", "tree", "any"][int(r.integers(0, 4))]
    x = Call(dtype, lens, B, Hq, Hkv, int(r.choice([64, 128])), int(r.choice([16, 32, 64, 128, 512])), counts, mode, seed=seed, strided=bool(r.integers(0, 2)))
    x.check(x.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests(dtype):
    """More requests than a wavefront has lanes, most of them short, some without rows or tokens."""
    r = np.random.default_rng(3)
    N = 150
    lens = [int(r.integers(0, 60)) for _ in range(N)]
    lens[70], lens[149], lens[64] = 3000, 1500, 0
    counts = [int(r.integers(0, 3)) for _ in range(N)]
    counts[149] = 2
    x = Call(dtype, lens, 2, 8, 2, 64, 16, counts, "causal", seed=4)
    x.check(x.run())


def test_a_long_cache():
    x = Call("bf16", [100003, 5], 2, 8, 1, 128, 64, None, "causal", seed=5)
    x.check(x.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hq", [(8, 28), (5, 8), (13, 28), (9, 64)])
def test_more_pieces_than_compute_units(dtype, B, Hq):
    """Wavefronts of the second workgroups on a compute unit may have other rows; M-tiles of one to four wavefronts and of two M-tiles."""
    x = Call(dtype, [2500, 1999, 2111, 64, 3000, 2345], B, Hq, 4, 128, 16, [B, B, B - 2, B, B, 1], "tree", seed=B)
    x.check(x.run())


def test_pages_beyond_32_bits():
    """A pool of 5 GB: the request's pages lie behind the first 2^32 bytes, and the same ones in front of them give the same result."""
    x = Call("bf16", [150, 3], 3, 8, 2, 128, 64, None, "causal", seed=9)
    want = x.run()
    small, used = x.cache, x.cache.k.shape[0]
    pages = (5 << 30) // (2 * 64 * 128 * 2)
    k, v = (torch.empty((pages,) + tuple(t.shape[1:]), dtype=t.dtype, device="cuda") for t in (small.k, small.v))
    k[-used:], v[-used:] = small.k, small.v
    table = small.page_table.clone()
    table[(table >= 0) & (table < used)] += pages - used
    x.cache = F.PagedCache(k, v, table, small.lens)
    assert torch.equal(x.run(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_entries_that_name_no_page(dtype):
    """They are read as the nearest page there is."""
    x = Call(dtype, [200, 90], 5, 8, 2, 64, 16, None, "causal", seed=10)
    pages = x.cache.k.shape[0]
    for t in (x.cache.k, x.cache.v):
        t.nan_to_num_(0.5)
    good, bad = x.cache.page_table.clone(), x.cache.page_table.clone()
    good[0, 3], good[0, 12], good[1, 0] = 0, pages - 1, pages - 1
    bad[0, 3], bad[0, 12], bad[1, 0] = -1, pages, 2 ** 31 - 1
    x.cache.page_table.copy_(good)
    want = x.run()
    x.cache.page_table.copy_(bad)
    assert torch.equal(x.run(), want)


def test_two_streams_at_once():
    """Calls side by side, each with a workspace of its own, give what they give alone."""
    a, b = (Call("bf16", [1500, 700], 8, 28, 4, 128, 16, None, "tree", seed=s) for s in (11, 12))
    want = [a.run(), b.run()]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, x in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(x.run())
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_stay(dtype):
    x = Call(dtype, [40, 700], 20, 14, 2, 64, 16, [7, 0], "tree", seed=6)
    out = torch.full_like(x.q.contiguous(), 3.0)
    assert x.run(out=out) is out
    x.check(out, untouched=3.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_beyond_the_table_and_max_len(dtype):
    x = Call(dtype, [200, 128, 64], 4, 8, 2, 64, 64, None, "causal", seed=7, extra_pages=0)
    x.check(x.run(max_len=100), max_len=100)
    x.check(x.run(max_len=1), max_len=1)
    x = Call(dtype, [256, 256], 4, 8, 2, 64, 64, None, "causal", seed=8, extra_pages=0)
    x.cache.lens.copy_(ints([1 << 30, -5]))
    x.lens = [256, 0]
    x.check(x.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_and_large_scores(dtype):
    x = Call(dtype, [300, 20], 9, 8, 2, 128, 32, None, "tree", seed=9, spread=4.0)
    x.check(x.run())                       # scores up to a few hundred: one key takes all
    x.check(x.run(scale=0.01), scale=0.01)
    x.check(x.run(scale=1.5), scale=1.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_hidden_keys_may_hold_anything(dtype):
    x = Call(dtype, [100], 6, 4, 2, 64, 16, None, "causal", seed=10)
    want = x.run().clone()
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(x.dtype).min):
        x.k[0, 5] = bad                    # only token 5 sees it
        got = x.run()
        assert torch.equal(got[0, :5], want[0, :5])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_mask_for_all_requests(dtype):
    x = Call(dtype, [100, 300, 0], 10, 4, 2, 64, 16, None, "tree", seed=11)
    x.mask = x.mask[0].contiguous()
    x.see = [x.see[0]] * 3
    x.check(x.run())


def test_streams_workspaces_and_graphs():
    """Two captured calls that share a workspace, replayed in turn while lens, pages and values change, against eager calls."""
    a = Call("bf16", [900, 130], 6, 28, 4, 128, 16, None, "tree", seed=12)
    b = Call("bf16", [64, 2000], 1, 28, 4, 128, 64, None, "full", seed=13)
    need = max(F.fdd_paged_attn_workspace(x.q, x.cache, x.k, x.v) for x in (a, b))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    counts = [ints(x.counts) for x in (a, b)]
    outs = [torch.zeros_like(x.q) for x in (a, b)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    for x, c, o in zip((a, b), counts, outs):
        x.run(out=o, workspace=ws, n_tokens=c, stream=s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            x.run(out=o, workspace=ws, n_tokens=c)
        graphs.append(g)
    for step in range(4):
        for x, c, o, g in zip((a, b), counts, outs, graphs):
            x.lens = [max(0, n - 70 * step) for n in x.lens]
            x.cache.lens.copy_(ints(x.lens))
            x.q.mul_(0.9)
            o.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            x.check(o)
            assert torch.equal(o, x.run())


def test_results_do_not_depend_on_the_run():
    x = Call("bf16", [5000, 100, 7], 8, 28, 4, 128, 16, None, "tree", seed=14)
    first = x.run().clone()
    for _ in range(5):
        assert torch.equal(x.run(), first)


def test_wrong_arguments():
    x = Call("bf16", [40], 4, 8, 2, 64, 16)
    with pytest.raises(ValueError):
        F.fdd_paged_attn(x.q[:, :, :, :32], x.cache, x.k, x.v)
    with pytest.raises(ValueError):
        F.fdd_paged_attn(x.q, x.cache, x.k[:, :3], x.v)
    with pytest.raises(TypeError):
        F.fdd_paged_attn(x.q.float(), x.cache, x.k, x.v)
    with pytest.raises(TypeError):
        F.fdd_paged_attn(x.q, x.cache, x.k, x.v, mask=torch.zeros(1, 4, 2, dtype=torch.int64, device="cuda"))
    with pytest.raises(TypeError):
        F.fdd_paged_attn(x.q, x.cache, x.k, x.v, n_tokens=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(F.FddError):
        F.fdd_paged_attn(x.q, x.cache, x.k, x.v, mask=torch.zeros(1, 4, 1, dtype=torch.int64, device="cuda"), causal_block=True)
    with pytest.raises(F.FddError):
        F.fdd_paged_attn(x.q, x.cache, x.k, x.v, out=x.q)
    with pytest.raises(ValueError):
        F.fdd_paged_attn(x.q, x.cache, x.k, x.v, workspace=torch.empty(1 << 20, dtype=torch.uint8))
    y = Call("bf16", [400], 4, 8, 2, 64, 16)
    with pytest.raises(F.FddError):
        y.run(workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
