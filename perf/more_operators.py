"""The operators of speculative decoding over a paged cache.

A case is one of five kinds of pass, each of them one use of the public Python entry points:

``rope``      positions are rotated into the queries and keys of a step or a prompt (``fdd_rope``)
``append``    rows of K and V join the pages of every request behind the rows it holds, keys rotated on the way or, behind a
              verification, the rows of the accepted path as they are (``fdd_paged_append``)
``tree``      what every drafted token may see, as bits, and its position, from the tree's parents (``fdd_tree_mask``)
``attn``      attention of every request's new tokens (one, a chain, a block or a tree) over its pages and one another
              (``fdd_paged_attn``)
``verify``    the drafted tokens that the target's probabilities let stand, from given random numbers, the token behind
              them, and the chance that each drafted token had (``fdd_tree_verify``)

Pages: K and V [pages, Hkv, page_size, D], the pages of request n listed in page_table[n], of which it holds lens[n] rows.
Trees: token 0 of a request is its last certain one, token i follows token parents[i] < i; without parents token i follows i - 1.

Where ``own`` is false the operators are worked out in elementary torch operations.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_DEFAULTS = dict(dtype="bf16", N=1, B=1, L=0, Hq=28, Hkv=4, D=128, page=64, ragged=False, mode="causal", rot=128, interleaved=False, base=1e6,
                 scaling="none", stretch=1.0, original=4096, first=0, rotate=True, path=False, V=0, draft=False, tree=False, temperature=1.0)


def _case(name=None, **kw):
    c = dict(_DEFAULTS)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one layer of a step of one request, a block of 32 tokens at the end of a long prompt: pure latency
        _case("rope_block", kind="rope", B=32, first=16384),
        # a prompt of several camera images in one piece, a cache stretched to four times the length that was trained
        _case("rope_prompt", kind="rope", B=16384, scaling="parts", stretch=4.0, original=32768, first=65536),
        # behind a verification: the accepted rows of 16 requests' trees join their pages, already rotated
        _case("append_path", kind="append", N=16, B=32, L=4000, ragged=True, page=16, rotate=False, path=True),
        # the prompts of four requests of uneven length are written at once, behind a shared system prompt
        _case("append_prompt", kind="append", N=4, B=8192, L=1000, ragged=True),
        # one request's tree of 16 drafted tokens
        _case("tree_one", kind="tree", N=1, B=16, L=4000),
        # many requests with large trees of uneven size
        _case("tree_batch", kind="tree", N=64, B=256, L=4000, ragged=True),
        # ordinary decoding: one token of each of 16 requests, caches of uneven length in small pages
        _case("attn_token", kind="attn", N=16, B=1, L=8192, ragged=True, page=16),
        # one layer of a verify pass: trees of 32 drafted tokens of four requests
        _case("attn_tree", kind="attn", N=4, B=32, L=4096, mode="tree"),
        # nothing a multiple of anything, in fp32 and with small heads: what a bf16 result is checked against
        _case("attn_ragged_f32", kind="attn", dtype="f32", N=3, B=21, L=2003, Hq=14, Hkv=2, D=64, ragged=True, mode="tree", page=32),
        # 16 requests with long caches, blocks of 64 tokens that see each other both ways
        _case("attn_long", kind="attn", N=16, B=64, L=16384, mode="full"),
        # a chain of 8 tokens that a small model drew from its own probabilities, an odd vocabulary in fp32
        _case("verify_chain_f32", kind="verify", dtype="f32", N=4, B=9, V=50001, draft=True),
        # trees of 32 tokens, the likeliest ones of a draft pass, over the model's vocabulary
        _case("verify_tree", kind="verify", N=8, B=32, V=152064, tree=True, temperature=0.7),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("flops", "bytes")}
    while True:
        kind = rng.choice(("rope", "append", "append", "tree", "attn", "attn", "attn", "attn", "verify", "verify"))
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        Hq, Hkv = rng.choice(((28, 4), (28, 4), (14, 2), (32, 8), (16, 4), (8, 8), (4, 1)))
        D = rng.choice((128, 128, 64))
        c = _case(kind=kind, dtype=dtype, Hq=Hq, Hkv=Hkv, D=D, page=rng.choice((16, 32, 64, 64, 128, 256)), ragged=rng.random() < 0.6)
        c.update(rot=rng.choice((D, D, D // 2, 24)), interleaved=rng.random() < 0.4, base=rng.choice((1e4, 1e6)))
        if rng.random() < 0.5:
            c.update(scaling=rng.choice(("linear", "base", "parts")), stretch=rng.choice((2.0, 4.0, 10.0)), original=rng.choice((4096, 32768)))
        if kind == "rope":
            c.update(N=_logint(rng, 1, 64), B=_logint(rng, 1, 16384), first=rng.choice((0, 1000, 131071, 1000003)))
        elif kind == "append":
            c.update(N=_logint(rng, 1, 64), B=_logint(rng, 1, 16384), L=rng.choice((0, 1, 63, rng.randrange(0, 5000))), rotate=rng.random() < 0.7)
            if c["B"] <= 256:
                c["path"] = rng.random() < 0.5
        elif kind == "tree":
            c.update(N=_logint(rng, 1, 64), B=_logint(rng, 1, 256), L=rng.randrange(0, 10000))
        elif kind == "attn":
            c.update(N=_logint(rng, 1, 64), B=rng.choice((1, 1, 2, 5, 8, 16, 31, 32, 64, 65, 128)), mode=rng.choice(("causal", "tree", "tree", "full")),
                     L=_logint(rng, 1, 32768) if rng.random() < 0.9 else 0)
        else:
            c.update(N=_logint(rng, 1, 32), B=rng.choice((1, 2, 5, 8, 9, 16, 32, 64)),
                     V=rng.choice((152064, 152064, 65536, 50001, 32768, 9973, 512, _logint(rng, 64, 152064))),
                     temperature=rng.choice((1.0, 1.0, 0.7, 0.0)))
            if rng.random() < 0.5:
                c["tree"] = True
            else:
                c["draft"] = c["temperature"] > 0.0 and rng.random() < 0.7
        w = work(c)
        if w["flops"] <= (15.3e9 if dtype == "f32" and kind == "attn" else most["flops"]) and w["bytes"] <= most["bytes"]:
            return c


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _lens(c):
    """Rows that each request holds before the pass: L of the longest, the others down to a quarter of it."""
    N, L = c["N"], c["L"]
    return [L - (L * 3 // 4) * ((5 * n) % N) // max(1, N - 1) if c["ragged"] and N > 1 else L for n in range(N)]


def _counts(c):
    """New tokens of each request: B of the first, the others down to half of it."""
    N, B = c["N"], c["B"]
    return [max(1, B - (B // 2) * ((3 * n) % N) // max(1, N - 1)) if c["ragged"] and N > 1 else B for n in range(N)]


def _parents(c, seed):
    """A random tree for each request; a token follows one of the few before it, so that paths of some length come up."""
    r = random.Random(seed * 1000003 + 17)
    return [[-1] + [max(0, i - 1 - int(r.expovariate(0.4))) for i in range(1, c["B"])] for _ in range(c["N"])]


def _paths(parents, counts, seed):
    """The path from token 0 to some token of each request's tree."""
    r = random.Random(seed * 7919 + 5)
    out = []
    for p, n in zip(parents, counts):
        i, path = r.randrange(n), []
        while i >= 0:
            path.append(i)
            i = p[i]
        out.append(path[::-1])
    return out


def _inputs(case, seed):
    """Everything that is drawn, from the seed alone."""
    c = dict(_DEFAULTS, **case)
    dev, dt = "cuda", _DTYPES[c["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=dev).normal_(0.0, 1.0, generator=g)

    def ints(rows):
        return torch.tensor(rows, dtype=torch.int32, device=dev)

    x = {"case": c}
    N, B, L, Hq, Hkv, D, page = (c[k] for k in ("N", "B", "L", "Hq", "Hkv", "D", "page"))
    lens, counts = _lens(c), _counts(c)
    x["lens"], x["counts"] = ints(lens), ints(counts)
    if c["kind"] == "rope":
        x["q"], x["k"] = normal(N, B, Hq, D), normal(N, B, Hkv, D)
        x["positions"] = (torch.arange(B, dtype=torch.int32, device=dev) + c["first"]).expand(N, B).contiguous()
        return x
    x["parents"] = ints(_parents(c, seed))
    if c["kind"] == "tree":
        return x
    if c["kind"] == "verify":
        V = c["V"]
        logits = torch.empty((N, B, V), dtype=torch.float32, device=dev).normal_(0.0, 2.0, generator=g)
        tok = torch.randint(0, V, (N, B), generator=g, device=dev)
        n_at = torch.arange(N, device=dev)[:, None].expand(N, B)
        if c["draft"]:
            # a small model that is near the target, and a chain of what it drew
            x["draft"] = (logits + torch.empty_like(logits).normal_(0.0, 0.5, generator=g)).to(dt)
            drawn = torch.multinomial(torch.softmax(x["draft"].view(N * B, V).float(), -1), 1, generator=g).view(N, B)
            tok[:, 1:] = drawn[:, :-1]
        elif B > 1:
            # drafted tokens are likely ones behind the token that they follow; no two behind the same one are alike
            follows = x["parents"].long() if c["tree"] else torch.arange(-1, B - 1, device=dev).expand(N, B)
            tok = (tok // 64 * 64 + torch.arange(B, device=dev) % 64) % V if V >= 128 and B <= 64 else tok
            logits[n_at[:, 1:], follows[:, 1:], tok[:, 1:]] += 11.0 + 3.0 * torch.rand((N, B - 1), generator=g, device=dev)
        # entries that a schema rules out
        ruled = torch.randint(0, V, (max(1, V // 64),), generator=g, device=dev)
        logits[:, ::3][..., ruled] = -math.inf
        x["logits"], x["tokens"] = logits.to(dt), tok.to(torch.int32)
        x["uniforms"] = torch.rand((N, B, 2), generator=g, device=dev)
        return x
    # pages: each request's lie anywhere among all of them
    rows = [max(1, (n + (B if c["kind"] == "append" else 0) + page - 1) // page) for n in lens]
    total, wide = sum(rows) + 3, max(rows) + 1
    order = torch.randperm(total, generator=g, device=dev).to(torch.int32)
    table, at = torch.zeros((N, wide), dtype=torch.int32, device=dev), 0
    for n in range(N):
        table[n, :rows[n]] = order[at:at + rows[n]]
        at += rows[n]
    x["table"] = table
    spread = (0.5 + 1.5 * torch.rand((Hkv, 1, D), generator=g, device=dev)).to(dt)        # channels of different spread
    x["k_pages"], x["v_pages"] = normal(total, Hkv, page, D) * spread, normal(total, Hkv, page, D)
    if c["kind"] == "append":
        # parts of one projection
        qkv = normal(N, B, (Hq + 2 * Hkv) * D) if B <= 256 else normal(N, B, 2 * Hkv * D)
        x["k"] = qkv[:, :, -2 * Hkv * D:-Hkv * D].unflatten(2, (Hkv, D))
        x["v"] = qkv[:, :, -Hkv * D:].unflatten(2, (Hkv, D))
        if c["path"]:
            paths = _paths(_parents(c, seed), counts, seed)
            x["rows"] = ints([p + [-1] * (B - len(p)) for p in paths])
            x["counts"] = ints([len(p) for p in paths])
        else:
            x["rows"] = None
        return x
    x["q"], x["bk"], x["bv"] = normal(N, B, Hq, D), normal(N, B, Hkv, D) * spread.transpose(0, 1), normal(N, B, Hkv, D)
    if c["mode"] == "tree":
        sees = np.zeros((N, B, (B + 63) // 64 * 64), dtype=bool)
        for n, p in enumerate(_parents(c, seed)):
            for i in range(counts[n]):
                if i:
                    sees[n, i] = sees[n, p[i]]
                sees[n, i, i] = True
        x["bits"] = torch.from_numpy(np.packbits(sees, axis=-1, bitorder="little").view(np.int64)).to(dev)
    else:
        x["bits"] = None
    return x


# ---- the plain form --------------------------------------------------------------------------------------------------

def _plain_angles(c):
    """Radians a position turns each pair of channels by, in 64 bits, and the factor of all rotated channels."""
    R, s = c["rot"], c["stretch"]
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    base, magnitude = c["base"], 1.0
    if c["scaling"] == "base":
        base = base * s ** (R / (R - 2))
    w = base ** (-2.0 * i / R)
    if c["scaling"] == "linear":
        w = w / s
    elif c["scaling"] == "parts":
        turns = c["original"] * w / (2.0 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        w = w * keep + w / s * (1.0 - keep)
        magnitude = 0.1 * math.log(s) + 1.0
    return w, magnitude


def _plain_rotate(c, x, positions):
    """x [..., heads, D] in 32 bits, positions [...]"""
    w, magnitude = _plain_angles(c)
    R = c["rot"]
    a = positions.double()[..., None] * w
    cos, sin = ((f(a) * magnitude).float()[..., None, :] for f in (torch.cos, torch.sin))
    y = x.float()
    if c["interleaved"]:
        u, v = y[..., 0:R:2], y[..., 1:R:2]
        turned = torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)
    else:
        u, v = y[..., :R // 2], y[..., R // 2:R]
        turned = torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
    return torch.cat([turned, y[..., R:]], -1)


def _plain_append(x):
    c = x["case"]
    B, page = c["B"], c["page"]
    j = torch.arange(B, device="cuda")[None, :]
    n = torch.arange(c["N"], device="cuda")[:, None].expand(-1, B)
    valid = j < x["counts"][:, None]
    slot = x["lens"].long()[:, None] + j
    src = j.expand(c["N"], -1) if x["rows"] is None else x["rows"].long()
    n, slot, src = n[valid], slot[valid], src[valid]
    k = _plain_rotate(c, x["k"][n, src], slot).to(x["k"].dtype) if c["rotate"] else x["k"][n, src]
    at = x["table"].long()[n, slot // page]
    x["k_pages"][at, :, slot % page] = k
    x["v_pages"][at, :, slot % page] = x["v"][n, src]
    return x["k_pages"], x["v_pages"]


def _plain_tree(x):
    c = x["case"]
    N, B = c["N"], c["B"]
    there = torch.arange(B, device="cuda")[None, :] < x["counts"][:, None]
    sees = torch.eye(B, dtype=torch.bool, device="cuda").expand(N, B, B).clone()
    rows, at = torch.arange(N, device="cuda"), x["parents"].long()
    for i in range(1, B):
        sees[:, i] |= sees[rows, at[:, i]]
    sees &= there[:, :, None]
    depth = (sees.sum(-1) - 1).clamp_min(0)
    wide = torch.zeros((N, B, (B + 63) // 64 * 64), dtype=torch.int64, device="cuda")
    wide[..., :B] = sees
    bits = (wide.view(N, B, -1, 64) << torch.arange(64, device="cuda")).sum(-1)
    return bits, (x["lens"][:, None] + depth.to(torch.int32)) * there


def _hidden(c, bits, n, count):
    """[count, count]: which of request n's new tokens a new token does not see."""
    i = torch.arange(count, device="cuda")
    if c["mode"] == "full":
        return torch.zeros((count, count), dtype=torch.bool, device="cuda")
    if c["mode"] == "causal":
        return i[None, :] > i[:, None]
    return (bits[n, :count][:, i // 64] >> (i % 64)[None, :]) & 1 == 0


def _plain_attn(x):
    c = x["case"]
    Hkv, D, G, page = c["Hkv"], c["D"], c["Hq"] // c["Hkv"], c["page"]
    for n, (L, count) in enumerate(zip(_lens(c), _counts(c))):
        pages = x["table"][n, :(L + page - 1) // page].long()
        kv = [torch.cat([p[pages].transpose(0, 1).reshape(Hkv, -1, D)[:, :L], b[n, :count].transpose(0, 1)], 1).float()
              for p, b in ((x["k_pages"], x["bk"]), (x["v_pages"], x["bv"]))]
        hidden = _hidden(c, x["bits"], n, count).repeat_interleave(G, 0)
        for h in range(Hkv):
            q = x["q"][n, :count, h * G:(h + 1) * G].reshape(count * G, D).float()
            s = q @ kv[0][h].T.contiguous() * (1.0 / math.sqrt(D))
            s[:, L:].masked_fill_(hidden, -math.inf)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            o = (p @ kv[1][h]) / p.sum(-1, keepdim=True)
            x["out"][n, :count, h * G:(h + 1) * G] = o.view(count, G, D).to(x["out"].dtype)
    return x["out"]


def _plain_verify(x):
    """Tokens in order: one that follows the last accepted one is tried, and is where the walk goes on if it stands."""
    c = x["case"]
    N, B, V, t = c["N"], c["B"], c["V"], c["temperature"]
    path, taken, emitted, chances = x["out"]
    path.fill_(-1)
    emitted.fill_(-1)
    rows, ids = torch.arange(N, device="cuda"), torch.arange(V, device="cuda")
    parents = x["parents"] if c["tree"] else torch.arange(-1, B - 1, device="cuda").expand(N, B)
    now = torch.zeros(N, dtype=torch.int64, device="cuda")
    steps = torch.zeros(N, dtype=torch.int64, device="cuda")
    path[:, 0] = 0

    def softmax(z, temperature):
        y = z[rows, now].double() / temperature       # (what is drawn lies next to borders)
        e = torch.exp(y - y.amax(-1, keepdim=True))
        return e / e.sum(-1, keepdim=True)

    def best():
        z = x["logits"][rows, now].float()
        return torch.where(z == z.amax(-1, keepdim=True), ids, V).amin(-1)

    if t > 0.0:
        p = softmax(x["logits"], t)
        w, out_of, total = p, torch.zeros(N, dtype=torch.float64, device="cuda"), torch.ones(N, dtype=torch.float64, device="cuda")
    for j in range(1, B):
        token = x["tokens"][:, j].long()
        tried = (parents[:, j] == now) & (j < x["counts"])
        if t == 0.0:
            stands = tried & (best() == token)
        else:
            q = softmax(x["draft"], 1.0) if x["draft"] is not None else None
            q_token = q[rows, token] if q is not None else 1.0
            stands = tried & (x["uniforms"][:, j, 0].double() * q_token * total < w[rows, token])
            falls = (tried & ~stands)[:, None]
            if q is not None:
                out_of = torch.where(falls[:, 0], out_of + total, out_of)
                w = torch.where(falls, (p - out_of[:, None] * q).clamp_min(0.0), w)
            else:
                w = torch.where(falls & (ids == token[:, None]), 0.0, w)
            total = torch.where(falls[:, 0], w.sum(-1), total)
        at = steps[:, None]
        emitted.scatter_(1, at, torch.where(stands, token, emitted.gather(1, at)[:, 0].long()).to(torch.int32)[:, None])
        now = torch.where(stands, j, now)
        steps = steps + stands
        at = steps[:, None]
        path.scatter_(1, at, torch.where(stands, j, path.gather(1, at)[:, 0].long()).to(torch.int32)[:, None])
        if t > 0.0:
            p = softmax(x["logits"], t)
            w = torch.where(stands[:, None], p, w)
            out_of, total = torch.where(stands, 0.0, out_of), torch.where(stands, 1.0, total)
    if t == 0.0:
        last = best()
    else:
        w = torch.where((total < 2.0 ** -40)[:, None], p, w)
        cum = w.cumsum(-1)
        over = cum <= x["uniforms"][rows, now, 1].double()[:, None] * cum[:, -1:]
        last = torch.minimum(over.sum(-1), torch.where(w > 0.0, ids, -1).amax(-1))
    emitted.scatter_(1, steps[:, None], last.to(torch.int32)[:, None])
    taken.copy_(steps + 1)
    # the chance of every token when it is tried first behind the one that it follows
    there = torch.arange(B, device="cuda") < x["counts"][:, None]
    chances.copy_(there)
    for i in range(1, B):
        now, token = parents[:, i].long(), x["tokens"][:, i].long()
        if t == 0.0:
            chance = (best() == token).double()
        else:
            chance = softmax(x["logits"], t)[rows, token]
            if x["draft"] is not None:
                chance = (chance / softmax(x["draft"], 1.0)[rows, token]).clamp_max(1.0)
        chances[:, i] = torch.where(there[:, i], chance, 0.0).float()
    return path, taken, emitted, chances


# ---- one pass -----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    x = _inputs(case, seed)
    c = x["case"]
    kind, N, B = c["kind"], c["N"], c["B"]
    x["ws"], x["turns"] = None, None
    if own:
        import paper_2605_23163_amd as F
    if own and (kind == "rope" or kind == "append" and c["rotate"]):
        how = {} if c["scaling"] == "none" else dict(scaling=c["scaling"], stretch=c["stretch"], original=c["original"])
        x["turns"] = F.fdd_rope_table(c["rot"], base=c["base"], interleaved=c["interleaved"], **how)
    if kind == "rope":
        x["out"] = (torch.empty_like(x["q"]), torch.empty_like(x["k"]))
    elif kind == "tree":
        x["out"] = (torch.zeros((N, B, (B + 63) // 64), dtype=torch.int64, device="cuda"), torch.zeros((N, B), dtype=torch.int32, device="cuda"))
    elif kind == "attn":
        x["out"] = torch.zeros_like(x["q"])
    elif kind == "verify":
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        x["out"] = (z(N, B), z(N), z(N, B), torch.zeros((N, B), dtype=torch.float32, device="cuda"))
        x.setdefault("draft", None)
        if not c["tree"]:
            x["parents"] = None
    if own and kind in ("append", "attn"):
        x["cache"] = F.PagedCache(x["k_pages"], x["v_pages"], x["table"], x["lens"])
    if own and kind == "attn":
        x["ws"] = torch.empty(max(256, F.fdd_paged_attn_workspace(x["q"], x["cache"], x["bk"], x["bv"])), dtype=torch.uint8, device="cuda")
    if own and kind == "verify":
        x["ws"] = torch.empty(max(256, F.fdd_tree_verify_workspace(x["logits"], x["draft"])), dtype=torch.uint8, device="cuda")
    return x


def run(x):
    c = x["case"]
    kind = c["kind"]
    if own:
        import paper_2605_23163_amd as F
        if kind == "rope":
            return F.fdd_rope(x["q"], x["positions"], x["turns"], k=x["k"], out=x["out"][0], k_out=x["out"][1])
        if kind == "append":
            F.fdd_paged_append(x["k"], x["v"], x["cache"], table=x["turns"], rows=x["rows"], n_rows=x["counts"])
            return x["cache"].k, x["cache"].v
        if kind == "tree":
            return F.fdd_tree_mask(x["parents"], lens=x["lens"], n_tokens=x["counts"], mask=x["out"][0], positions=x["out"][1])
        if kind == "attn":
            return F.fdd_paged_attn(x["q"], x["cache"], x["bk"], x["bv"], mask=x["bits"], n_tokens=x["counts"], causal_block=c["mode"] == "causal",
                                    out=x["out"], workspace=x["ws"])
        return F.fdd_tree_verify(x["logits"], x["tokens"], x["uniforms"], parents=x["parents"], draft_logits=x["draft"], n_tokens=x["counts"],
                                 temperature=c["temperature"], path=x["out"][0], n_path=x["out"][1], emitted=x["out"][2], chances=x["out"][3],
                                 workspace=x["ws"])
    if kind == "rope":
        for o, t in zip(x["out"], (x["q"], x["k"])):
            o.copy_(_plain_rotate(c, t, x["positions"]))
        return x["out"]
    return {"append": _plain_append, "tree": _plain_tree, "attn": _plain_attn, "verify": _plain_verify}[kind](x)


def work(case):
    """Every input read once and every output written once."""
    c = dict(_DEFAULTS, **case)
    es = 2 if c["dtype"] == "bf16" else 4
    N, B, Hq, Hkv, D = (c[k] for k in ("N", "B", "Hq", "Hkv", "D"))
    lens, counts = _lens(c), _counts(c)
    if c["kind"] == "rope":
        return {"bytes": N * B * ((Hq + Hkv) * D * es * 2 + 4), "flops": 3.0 * N * B * (Hq + Hkv) * c["rot"]}
    if c["kind"] == "append":
        rows = sum(min(n, 6) for n in counts) if c["path"] else sum(counts)      # (an accepted path is a few tokens long)
        return {"bytes": rows * Hkv * D * es * 4 + N * 8, "flops": 3.0 * rows * Hkv * c["rot"] if c["rotate"] else 0.0}
    if c["kind"] == "tree":
        return {"bytes": N * (B * (4 + 8 * ((B + 63) // 64) + 4) + 8), "flops": 0.0}
    if c["kind"] == "verify":
        rows = sum(counts)
        return {"bytes": c["V"] * es * (2 * rows - N if c["draft"] else rows) + N * B * 28, "flops": 4.0 * rows * c["V"] * (2 if c["draft"] else 1)}
    seen = {"full": lambda n: n * n, "causal": lambda n: n * (n + 1) / 2, "tree": lambda n: n * (1 + min(n - 1, 6) / 2)}[c["mode"]]
    moved = sum(2 * (L + n) * Hkv * D * es + 2 * n * Hq * D * es for L, n in zip(lens, counts))
    return {"bytes": moved, "flops": sum(4.0 * Hq * D * (n * L + seen(n)) for L, n in zip(lens, counts))}


# ---- the operators from their definition, in 64 bits ----------------------------------------------------------------------

def _exact_rotate(c, x, positions):
    """Rows of heads [rows, heads, D] as complex numbers that are turned; positions [rows] on the host."""
    R, s = c["rot"], c["stretch"]
    base = c["base"] * (s ** (R / (R - 2)) if c["scaling"] == "base" else 1.0)
    w, size = [], 1.0
    for i in range(R // 2):
        f = math.exp(-2 * i / R * math.log(base))
        if c["scaling"] == "linear":
            f /= s
        if c["scaling"] == "parts":
            r = c["original"] * f / math.tau
            g = min(1.0, max(0.0, (r - 1) / (32 - 1)))
            f = (1 - g) * f / s + g * f
            size = 1 + math.log(s) / 10
        w.append(f)
    angle = np.outer(np.asarray(positions, dtype=np.longdouble), np.asarray(w, dtype=np.longdouble)) % (2 * np.longdouble(np.pi))
    turn = torch.polar(torch.full(angle.shape, size, dtype=torch.float64), torch.from_numpy(angle.astype(np.float64))).to(x.device)
    y = x.double().clone()
    z = y[..., :R].unflatten(-1, (R // 2, 2) if c["interleaved"] else (2, R // 2))
    z = z if c["interleaved"] else z.transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn[:, None])
    y[..., :R] = (z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2)
    return y


def exact(case, seed):
    x = _inputs(case, seed)
    c = x["case"]
    N, B, Hq, Hkv, D, page = (c[k] for k in ("N", "B", "Hq", "Hkv", "D", "page"))
    lens, counts = _lens(c), _counts(c)
    if c["kind"] == "rope":
        at = x["positions"].view(-1).cpu().numpy()
        return tuple(_exact_rotate(c, t.view(N * B, -1, D), at).view(t.shape) for t in (x["q"], x["k"]))
    if c["kind"] == "append":
        k, v = x["k_pages"].double(), x["v_pages"].double()
        table, held, wrote = x["table"].cpu().numpy(), x["lens"].tolist(), x["counts"].tolist()
        for n in range(N):
            src = torch.arange(wrote[n], device="cuda") if x["rows"] is None else x["rows"][n, :wrote[n]].long()
            at = held[n] + np.arange(wrote[n])
            kn, vn = x["k"][n].index_select(0, src).double(), x["v"][n].index_select(0, src).double()
            if c["rotate"]:
                kn = _exact_rotate(c, kn, at)
            pages, rows = torch.from_numpy(table[n, at // page]).long().cuda(), torch.from_numpy(at % page).cuda()
            k.transpose(1, 2)[pages, rows] = kn
            v.transpose(1, 2)[pages, rows] = vn
        return k, v
    if c["kind"] == "tree":
        words = np.zeros((N, B, (B + 63) // 64), dtype=np.uint64)
        places = np.zeros((N, B), dtype=np.int32)
        for n, p in enumerate(_parents(c, seed)):
            for i in range(counts[n]):
                a, places[n, i] = i, lens[n] - 1
                while a >= 0:
                    words[n, i, a >> 6] |= np.uint64(1 << (a & 63))
                    places[n, i] += 1
                    a = p[a]
        return words.view(np.int64), places
    if c["kind"] == "attn":
        out = torch.zeros((N, B, Hq, D), dtype=torch.float64, device="cuda")
        parents = _parents(c, seed)
        for n in range(N):
            L, m = lens[n], counts[n]
            add = torch.zeros((m, L + m), dtype=torch.float64)
            for i in range(m):
                seen = set(range(m)) if c["mode"] == "full" else set(range(i + 1))
                if c["mode"] == "tree":
                    a, seen = i, set()
                    while a >= 0:
                        seen.add(a)
                        a = parents[n][a]
                for j in range(m):
                    if j not in seen:
                        add[i, L + j] = -math.inf
            add = add.cuda()
            rows = torch.arange(L, device="cuda")
            where = x["table"][n].long()[rows // page]
            for h in range(Hkv):
                k = torch.cat([x["k_pages"][where, h, rows % page], x["bk"][n, :m, h]]).double()
                v = torch.cat([x["v_pages"][where, h, rows % page], x["bv"][n, :m, h]]).double()
                for hq in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    s = torch.mv if m == 1 else torch.mm
                    q = x["q"][n, :m, hq].double()
                    sc = s(k, q[0])[None] if m == 1 else s(q, k.T.contiguous())
                    out[n, :m, hq] = torch.softmax(sc / math.sqrt(D) + add, -1) @ v
        return out
    # verify: the same decisions from the definition, in logarithms
    V, t = c["V"], c["temperature"]
    parents = _parents(c, seed) if c["tree"] else [[i - 1 for i in range(B)] for _ in range(N)]
    path, emitted = (np.full((N, B), -1, dtype=np.int32) for _ in range(2))
    taken = np.zeros(N, dtype=np.int32)
    chances = np.zeros((N, B), dtype=np.float64)
    for n in range(N):
        chances[n, 0] = 1.0
        for i in sorted({parents[n][j] for j in range(1, counts[n])}):
            rows = [x["logits"][n, i].double() / (t or 1.0)] + ([x["draft"][n, i].double()] if c["draft"] else [])
            z = [r - torch.logsumexp(r, 0) for r in rows]
            for j in range(1, counts[n]):
                if parents[n][j] == i:
                    of = int(x["tokens"][n, j])
                    if t == 0.0:
                        chances[n, j] = float(of == int(torch.nonzero(rows[0] == rows[0].max())[0]))
                    else:
                        chances[n, j] = min(1.0, math.exp(float(z[0][of]) - (float(z[1][of]) if c["draft"] else 0.0)))
    tok, u = x["tokens"].cpu().numpy(), x["uniforms"].cpu().numpy().astype(np.float64)
    for n in range(N):
        i, k = 0, 0
        while True:
            path[n, k] = i
            kids = [j for j in range(counts[n]) if parents[n][j] == i and j != i]
            row = x["logits"][n, i].double().cpu().numpy()
            go = -1
            if t == 0.0:
                token = int(np.argmax(row))
                go = next((j for j in kids if tok[n, j] == token), -1)
            else:
                y = row / t
                left = np.exp(y - (y.max() + math.log(np.exp(y - y.max()).sum())))
                whole = left.copy()
                if c["draft"]:
                    z = x["draft"][n, i].double().cpu().numpy()
                    q = np.exp(z - (z.max() + math.log(np.exp(z - z.max()).sum())))
                for j in kids:
                    chance = left[tok[n, j]] / (q[tok[n, j]] if c["draft"] else 1.0) / (left.sum() or 1.0)
                    if u[n, j, 0] < chance:
                        go = j
                        break
                    if c["draft"]:
                        left = np.maximum(left / left.sum() - q, 0.0)
                    else:
                        left[tok[n, j]] = 0.0
                if go < 0:
                    if left.sum() < 2.0 ** -40:
                        left = whole
                    cum = np.cumsum(left)
                    token = int(np.searchsorted(cum, u[n, i, 1] * cum[-1], side="right"))
                    token = min(token, int(np.flatnonzero(left)[-1]))
            if go < 0:
                emitted[n, k] = token
                break
            emitted[n, k] = tok[n, go]
            i, k = go, k + 1
        taken[n] = k + 1
    return path, taken, emitted, chances
