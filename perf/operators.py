"""The operators of a prefix cache held in 8 bits, and the log probabilities of what a step writes.

A case is one of four kinds of pass, each of them one use of the public Python entry points:

``write``     K and V rows join the cache behind the rows it holds (``fdd_prefix_quantize``) and the rows of the blocks
              that this touched are read back (``fdd_prefix_dequantize``)
``read``      rows of a cache are read back
``attn``      attention of forked rollouts over a cache (``fdd_block_attn_quant``, for a batch of requests with a cache each
              ``fdd_block_attn_quant_batched``)
``logprobs``  log probability of a given token, entropy and top alternatives of every selected row of logits
              (``fdd_token_logprobs``)

The cache: K and V as e4m3, [Hkv, capacity, D], and a scale for each 64 rows of a head, [Hkv, capacity / 64], which is the
smallest power of two that brings the largest value of these rows to 448 or less (2^-117 at least, 2^119 at most).  A scale
only grows while rows join a block that has some; the rows there are rounded again where it does.

Where ``own`` is false the operators are worked out in elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 64
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_DEFAULTS = dict(dtype="bf16", N=1, B=32, L=2048, Hq=28, Hkv=4, D=128, E=0, problems=1, causal=False, only_values=False,
                 row0=0, rows=0, V=0, top=0, share=1.0, temperature=1.0)


def _case(name=None, **kw):
    c = dict(_DEFAULTS)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a finished block of 32 tokens joins the cache of its request, whose last block of rows is partly full: pure latency
        _case("write_block", kind="write", row0=4077, rows=32),
        # the prompt of a multi-camera request is written once, and read back whole
        _case("write_prompt", kind="write", rows=16384),
        # a piece of a cache of a small model in fp32, neither end of it at a block's: what a check or a tool reads
        _case("read_ragged_f32", kind="read", dtype="f32", Hkv=2, D=64, row0=1003, rows=5003),
        # one layer of the batch-1 decoder on the vehicle, short prompt
        _case("attn_n1", kind="attn", N=1, B=32, L=2048),
        # one layer of test-time scaling with 8 rollouts on one prefix
        _case("attn_n8", kind="attn", N=8, B=32, L=4096),
        # nothing a multiple of anything: head size 64, ragged prefix and block, an extension, rows of the value positions only
        _case("attn_ragged_d64", kind="attn", N=5, B=40, L=5003, Hq=14, Hkv=2, D=64, E=37, only_values=True),
        # requests in flight: 8 batch-1 problems in one launch, each with a long prefix of its own
        _case("attn_batched", kind="attn", N=1, B=32, L=16384, problems=8),
        # the long-prefix workload of the benchmark, 16 rollouts of 64 tokens, in the causal form of the verify pass
        _case("attn_n16", kind="attn", N=16, B=64, L=16384, causal=True),
        # the fp32 form of a step on a small model: what a bf16 result is checked against
        _case("attn_f32", kind="attn", dtype="f32", N=2, B=32, L=2048, Hq=14, Hkv=2, D=64),
        # the smallest head: a tiny block over a small vocabulary in fp32
        _case("logprobs_tiny_f32", kind="logprobs", dtype="f32", N=1, B=8, V=512, top=4),
        # one block of one request over an odd vocabulary, sampled tokens, as many alternatives as a client may ask for
        _case("logprobs_n1", kind="logprobs", N=1, B=32, V=50001, top=20, temperature=0.7),
        # 8 rollouts over the model's vocabulary, half of the block is scaffold and is not scored
        _case("logprobs_n8", kind="logprobs", N=8, B=32, V=152064, top=5, share=0.5),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("flops", "bytes")}
    while True:
        kind = rng.choice(("write", "write", "read", "attn", "attn", "attn", "attn", "logprobs", "logprobs"))
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        Hq, Hkv = rng.choice(((28, 4), (28, 4), (14, 2), (32, 8), (16, 4), (8, 8), (4, 1)))
        c = _case(kind=kind, dtype=dtype, Hq=Hq, Hkv=Hkv, D=rng.choice((128, 128, 64)))
        if kind in ("write", "read"):
            c["rows"] = _logint(rng, 1, 32768)
            c["row0"] = rng.choice((0, 64 * rng.randrange(0, 65), rng.randrange(0, 4097)))
        elif kind == "logprobs":
            c.update(N=_logint(rng, 1, 32), B=rng.choice((1, 4, 8, 20, 31, 32, 40, 64)),
                     V=rng.choice((152064, 152064, 65536, 50001, 32768, 9973, 512, _logint(rng, 64, 152064))),
                     top=rng.choice((0, 1, 4, 5, 8, 20)), share=rng.choice((1.0, 1.0, 0.7, 0.5)), temperature=rng.choice((1.0, 1.0, 0.7)))
        else:
            c.update(N=_logint(rng, 1, 32), B=rng.choice((1, 8, 31, 32, 32, 40, 64, 65, 96)),
                     L=64 * rng.randrange(1, 257) if rng.random() < 0.5 else _logint(rng, 1, 32768), E=rng.choice((0, 0, 0, 37, 64)),
                     causal=rng.random() < 0.3)
            if dtype == "bf16" and rng.random() < 0.25:
                c["problems"] = _logint(rng, 2, 16)
            elif rng.random() < 0.25:
                c["only_values"] = True
        w = work(c)
        if w["flops"] <= (15.3e9 if dtype == "f32" and kind == "attn" else most["flops"]) and w["bytes"] <= most["bytes"]:
            return c


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _capacity(c):
    held = c["L"] if c["kind"] == "attn" else c["row0"] + c["rows"]
    return (held + BLOCK - 1) // BLOCK * BLOCK + BLOCK


def _positions(c, g):
    """Value positions of a block (three of ten are scaffold), the same in every rollout: flat positions n B + b, ascending."""
    B, N = c["B"], c["N"]
    keep = torch.sort(torch.randperm(B, generator=g, device="cuda")[: max(1, B - int(round(0.3 * B)))]).values
    return (torch.arange(N, device="cuda")[:, None] * B + keep[None, :]).reshape(-1).to(torch.int32).contiguous()


def _value_count(c):
    return max(1, c["B"] - int(round(0.3 * c["B"]))) if c["only_values"] else c["B"]


def _inputs(case, seed):
    """Everything that is drawn, from the seed alone."""
    c = dict(_DEFAULTS, **case)
    dev, dt = "cuda", _DTYPES[c["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=dev).normal_(0.0, 1.0, generator=g)

    def keys(*shape, dtype):
        # keys have channels of different spread
        return normal(*shape, dtype=dtype) * (0.5 + 1.5 * torch.rand(shape[-2:], generator=g, device=dev)).to(dtype)

    x = {"case": c}
    Hkv, D, cap = c["Hkv"], c["D"], _capacity(c)
    if c["kind"] == "logprobs":
        N, B, V = c["N"], c["B"], c["V"]
        logits = torch.empty((N * B, V), dtype=torch.float32, device=dev).normal_(0.0, 2.0, generator=g)
        hit = torch.rand(N * B, generator=g, device=dev) < 0.3
        at = torch.randint(0, V, (N * B,), generator=g, device=dev)
        logits[torch.arange(N * B, device=dev), at] += 12.0 * hit.float()
        # entries that a schema rules out
        out = torch.randint(0, V, (max(1, V // 64),), generator=g, device=dev)
        logits[::3, out] = -math.inf
        x["logits"] = logits.to(dt).view(N, B, V)
        given = torch.randint(0, V, (N * B,), generator=g, device=dev)
        given = torch.where(torch.rand(N * B, generator=g, device=dev) < 0.5, at, given)
        ruled_out = logits.gather(1, given[:, None])[:, 0] == -math.inf
        x["tokens"] = torch.where(ruled_out, logits.argmax(-1), given).to(torch.int32).view(N, B)
        x["mask"] = None
        if c["share"] < 1.0:
            sel = torch.zeros(B, dtype=torch.uint8, device=dev)
            sel[torch.randperm(B, generator=g, device=dev)[: max(1, int(round(c["share"] * B)))]] = 1
            x["mask"] = sel.expand(N, B).contiguous()
        return x
    if c["kind"] == "attn":
        N, B, L, Hq, E, P = (c[k] for k in ("N", "B", "L", "Hq", "E", "problems"))
        q = [normal(N, B, Hq, D) for _ in range(P)]
        rows = [(keys(L, Hkv, D, dtype=torch.float32), normal(L, Hkv, D, dtype=torch.float32)) for _ in range(P)]
        bk, bv = [normal(N, B, Hkv, D) for _ in range(P)], [normal(N, B, Hkv, D) for _ in range(P)]
        ek, ev = ([normal(N, E + 3, Hkv, D) for _ in range(P)] for _ in range(2)) if E else (None, None)
        join = (lambda t: torch.stack(t)) if P > 1 else (lambda t: t[0])
        x.update(q=join(q), block_k=join(bk), block_v=join(bv), ext_k=join(ek) if E else None, ext_v=join(ev) if E else None)
        x["rows"] = rows
        x["positions"] = _positions(c, g) if c["only_values"] else None
        return x
    # a cache that holds rows up to row0 (write) or up to its last one (read); values of a block have a spread of their own
    held = c["row0"] if c["kind"] == "write" else c["row0"] + c["rows"]
    spread = torch.exp2(torch.randint(-2, 3, (cap // BLOCK, 1, 1), generator=g, device=dev).float()).repeat_interleave(BLOCK, 0)
    x["held"] = tuple(t * spread[:held] for t in (keys(held, Hkv, D, dtype=torch.float32), normal(held, Hkv, D, dtype=torch.float32)))
    if c["kind"] == "write":
        more = spread[c["row0"]:c["row0"] + c["rows"]].to(dt)
        x["k"], x["v"] = keys(c["rows"], Hkv, D, dtype=dt) * more, normal(c["rows"], Hkv, D) * more
    return x


# ---- the cache in its plain form -------------------------------------------------------------------------------------

def _scale_of(largest):
    """The smallest power of two s with largest / s <= 448 = 1.75 * 2^8, within [2^-117, 2^119]."""
    m, e = torch.frexp(largest)          # largest = m 2^e, m in [1/2, 1)
    e = e - 9 + (m > 0.875).to(e.dtype)
    e = torch.where(largest > 0, e, torch.full_like(e, -117))
    return torch.ldexp(torch.ones_like(largest), e.clamp(-117, 119))


def _codes(x, scale):
    """x / scale in e4m3, to the nearest and to even on ties (a division by a power of two: exact)."""
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _plain_write(codes, scales, x, row0):
    """Rows x [n, Hkv, D] join codes [Hkv, capacity, D] and scales [Hkv, capacity / 64] at row0."""
    n, Hkv, D = x.shape
    t0, t1 = row0 // BLOCK, (row0 + n + BLOCK - 1) // BLOCK
    lead = row0 - t0 * BLOCK
    y = torch.zeros((Hkv, (t1 - t0) * BLOCK, D), dtype=torch.float32, device=x.device)
    y[:, lead:lead + n] = x.float().transpose(0, 1)
    s = _scale_of(y.view(Hkv, t1 - t0, BLOCK * D).abs().amax(-1))
    if lead:
        s[:, 0] = torch.maximum(s[:, 0], scales[:, t0])
        y[:, :lead] = codes[:, t0 * BLOCK:row0].float() * scales[:, t0, None, None]
    c = _codes(y.view(Hkv, t1 - t0, BLOCK, D), s[:, :, None, None]).view(Hkv, -1, D)
    codes[:, t0 * BLOCK:row0 + n] = c[:, :lead + n]
    scales[:, t0:t1] = s


def _plain_read(codes, scales, row0, rows, dtype):
    """Rows [row0, row0 + rows) as they stand, [rows, Hkv, D]."""
    s = scales.repeat_interleave(BLOCK, 1)[:, row0:row0 + rows]
    return (codes[:, row0:row0 + rows].float() * s[:, :, None]).transpose(0, 1).to(dtype).contiguous()


def _empty_cache(c):
    Hkv, D, cap = c["Hkv"], c["D"], _capacity(c)
    lead = (c["problems"],) if c["problems"] > 1 else ()
    codes = [torch.zeros(lead + (Hkv, cap, D), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    scales = [torch.ones(lead + (Hkv, cap // BLOCK), dtype=torch.float32, device="cuda") for _ in range(2)]
    return codes + scales                # k, v, k_scale, v_scale


def prepare(case, seed):
    x = _inputs(case, seed)
    c = x["case"]
    if c["kind"] == "logprobs":
        N, B, K = c["N"], c["B"], c["top"]
        z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")
        x["out"] = (z(N, B), z(N, B), z(N, B, K, dtype=torch.int32), z(N, B, K))
        x["ws"] = None
        if own:
            import paper_2605_23163_amd as F
            x["ws"] = torch.empty(max(256, F.fdd_token_logprobs_workspace(x["logits"], top=K)), dtype=torch.uint8, device="cuda")
        return x
    cache = _empty_cache(c)
    held = x.pop("rows") if c["kind"] == "attn" else [x.pop("held")]
    for i, kv in enumerate(held):
        for j in range(2):
            if kv[j].shape[0]:
                at = (cache[j][i], cache[2 + j][i]) if c["problems"] > 1 else (cache[j], cache[2 + j])
                _plain_write(*at, kv[j], 0)
    x["cache"] = tuple(cache)
    if c["kind"] == "attn":
        x["out"] = torch.zeros_like(x["q"])
        x["ws"] = None
        if own:
            import paper_2605_23163_amd as F
            x["cache"] = F.QuantPrefix(*cache)
            kw = dict(ext_k=x["ext_k"], ext_v=x["ext_v"], E=c["E"]) if c["E"] else {}
            if c["problems"] > 1:
                need = F.fdd_block_attn_quant_batched_workspace(x["q"], x["cache"], c["L"], x["block_k"], x["block_v"], **kw)
            else:
                if c["only_values"]:
                    kw["n_q_positions"] = x["positions"].numel()
                need = F.fdd_block_attn_quant_workspace(x["q"], x["cache"], c["L"], x["block_k"], x["block_v"], **kw)
            x["ws"] = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    else:
        first = c["row0"] // BLOCK * BLOCK if c["kind"] == "write" else c["row0"]
        x["first"], x["count"] = first, c["row0"] + c["rows"] - first
        shape = (x["count"], c["Hkv"], c["D"])
        x["back"] = tuple(torch.empty(shape, dtype=_DTYPES[c["dtype"]], device="cuda") for _ in range(2))
        if own:
            import paper_2605_23163_amd as F
            x["cache"] = F.QuantPrefix(*cache)
    return x


# ---- one pass -----------------------------------------------------------------------------------------------------------

def _attend(c, q, cache, bk, bv, ek, ev, positions, out):
    """One problem: every rollout's queries against the prefix, its extension and its block, in fp32."""
    N, B, L, Hq, Hkv, D, E = (c[k] for k in ("N", "B", "L", "Hq", "Hkv", "D", "E"))
    G = Hq // Hkv
    rows = positions if positions is not None else torch.arange(N * B, device=q.device)
    per = rows.numel() // N              # positions of a rollout, the same number in each
    b = (rows.long() % B)
    pre = [_plain_read(cache[j], cache[2 + j], 0, L, torch.float32) for j in range(2)]
    qs = q.reshape(N * B, Hq, D)[rows.long()].float().view(N, per, Hq, D)
    res = torch.empty_like(qs)
    ahead = torch.arange(B, device=q.device)
    for n in range(N):
        parts = [[p, *([e[n, :E].float()] if E else []), blk[n].float()] for p, e, blk in zip(pre, (ek, ev), (bk, bv))]
        k, v = torch.cat(parts[0]), torch.cat(parts[1])
        hidden = (ahead[None, :] > b[n * per:(n + 1) * per, None]) if c["causal"] else None
        for h in range(Hkv):
            s = qs[n, :, h * G:(h + 1) * G].reshape(per * G, D) @ k[:, h].T.contiguous() * (1.0 / math.sqrt(D))
            if hidden is not None:
                s[:, L + E:].masked_fill_(hidden.repeat_interleave(G, 0), -math.inf)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            res[n, :, h * G:(h + 1) * G] = ((p @ v[:, h].contiguous()) / p.sum(-1, keepdim=True)).view(per, G, D)
    out.view(N * B, Hq, D)[rows.long()] = res.view(N * per, Hq, D).to(out.dtype)
    return out


def _plain_logprobs(x):
    c = x["case"]
    lp, ent, ids, tlp = x["out"]
    V, K = c["V"], c["top"]
    sel = torch.arange(c["N"] * c["B"], device="cuda") if x["mask"] is None else torch.nonzero(x["mask"].reshape(-1)).reshape(-1)
    z = x["logits"].view(-1, V)[sel].float()
    tok = x["tokens"].reshape(-1)[sel].long()
    m = z.amax(-1, keepdim=True)
    y = (z - m).double() / c["temperature"]       # (the sum runs over up to 2^17 entries)
    lse = torch.log(torch.exp(y).sum(-1, keepdim=True))
    logp = y - lse
    p = torch.exp(logp)
    lp.view(-1)[sel] = logp.gather(1, tok[:, None])[:, 0].float()
    ent.view(-1)[sel] = (-(p * torch.where(p > 0, logp, torch.zeros_like(logp))).sum(-1)).float()
    at = torch.arange(V, device="cuda")
    left = z.clone()
    for j in range(K):
        best = left.amax(-1, keepdim=True)
        i = torch.where(left == best, at, V).amin(-1)
        ids.view(-1, K)[sel, j] = i.to(torch.int32)
        tlp.view(-1, K)[sel, j] = logp.gather(1, i[:, None])[:, 0].float()
        left.scatter_(1, i[:, None], -math.inf)
    return x["out"]


def run(x):
    c = x["case"]
    kind = c["kind"]
    if own:
        import paper_2605_23163_amd as F
        if kind == "logprobs":
            lp, ent, ids, tlp = x["out"]
            return F.fdd_token_logprobs(x["logits"], x["tokens"], mask=x["mask"], top=c["top"], temperature=c["temperature"], logprobs=lp,
                                        entropy=ent, top_ids=ids, top_logprobs=tlp, workspace=x["ws"])
        cache = x["cache"]
        if kind == "attn":
            kw = dict(ext_k=x["ext_k"], ext_v=x["ext_v"], E=c["E"]) if c["E"] else {}
            if c["problems"] > 1:
                return F.fdd_block_attn_quant_batched(x["q"], cache, c["L"], x["block_k"], x["block_v"], out=x["out"], workspace=x["ws"],
                                                      causal_block=c["causal"], **kw)
            return F.fdd_block_attn_quant(x["q"], cache, c["L"], x["block_k"], x["block_v"], out=x["out"], workspace=x["ws"],
                                          causal_block=c["causal"], q_positions=x["positions"], **kw)
        if kind == "write":
            F.fdd_prefix_quantize(x["k"], x["v"], cache, row0=c["row0"])
        k, v = F.fdd_prefix_dequantize(cache, x["count"], row0=x["first"], k=x["back"][0], v=x["back"][1])
        return (k, v, cache.k_scale, cache.v_scale) if kind == "write" else (k, v)
    if kind == "logprobs":
        return _plain_logprobs(x)
    cache = x["cache"]
    if kind == "attn":
        args = [x[k] for k in ("q", "cache", "block_k", "block_v", "ext_k", "ext_v")]
        if c["problems"] > 1:
            for i in range(c["problems"]):
                q, ca, bk, bv, ek, ev = (t if t is None else [u[i] for u in t] if isinstance(t, tuple) else t[i] for t in args)
                _attend(c, q, ca, bk, bv, ek, ev, None, x["out"][i])
            return x["out"]
        return _attend(c, *args, x["positions"], x["out"])
    if kind == "write":
        _plain_write(cache[0], cache[2], x["k"], c["row0"])
        _plain_write(cache[1], cache[3], x["v"], c["row0"])
    for j in range(2):
        x["back"][j].copy_(_plain_read(cache[j], cache[2 + j], x["first"], x["count"], _DTYPES[c["dtype"]]))
    return (*x["back"], cache[2], cache[3]) if kind == "write" else x["back"]


def work(case):
    """Every input read once and every output written once."""
    c = dict(_DEFAULTS, **case)
    es = 2 if c["dtype"] == "bf16" else 4
    N, B, L, Hq, Hkv, D, E, P = (c[k] for k in ("N", "B", "L", "Hq", "Hkv", "D", "E", "problems"))
    if c["kind"] in ("write", "read"):
        first = c["row0"] // BLOCK * BLOCK if c["kind"] == "write" else c["row0"]
        n, held = c["row0"] + c["rows"] - first, c["row0"] - first
        blocks = (c["row0"] + c["rows"] + BLOCK - 1) // BLOCK - first // BLOCK
        # read back: codes and scales to values; written: values to codes and scales, behind what a block held
        moved = n * Hkv * D * (1 + es) + blocks * Hkv * 4
        if c["kind"] == "write":
            moved += c["rows"] * Hkv * D * (1 + es) + held * Hkv * D + blocks * Hkv * 4
        return {"bytes": 2 * moved, "flops": 2.0 * n * Hkv * D * (2 if c["kind"] == "write" else 1)}
    if c["kind"] == "logprobs":
        rows = N * (max(1, int(round(c["share"] * B))) if c["share"] < 1.0 else B)
        return {"bytes": rows * (c["V"] * es + 12 + 8 * c["top"]) + (N * B if c["share"] < 1.0 else 0), "flops": 6.0 * rows * c["V"]}
    pos = N * _value_count(c)
    blocks = (L + BLOCK - 1) // BLOCK
    kv = 2 * L * Hkv * D + 2 * blocks * Hkv * 4 + 2 * N * (E + B) * Hkv * D * es
    seen = pos * (L + E) + (N * B * (B + 1) / 2 if c["causal"] and not c["only_values"] else pos * (B + 1) / 2 if c["causal"] else pos * B)
    return {"bytes": P * (kv + 2 * pos * Hq * D * es), "flops": P * 4.0 * Hq * D * seen}


# ---- the operators from their definition, in 64 bits ----------------------------------------------------------------------

def _nearest(x, s):
    """The multiple of s by an e4m3 number that is nearest to x, the even one of two."""
    a = x / s
    step = torch.exp2(torch.floor(torch.log2(a.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(a / step).mul(step).clamp(-448, 448) * s


def _exact_scales(x):
    """[n rows of whole blocks, Hkv, D] -> [blocks, Hkv]"""
    top = x.abs().view(-1, BLOCK, *x.shape[1:]).amax((1, 3))
    e = torch.ceil(torch.log2(top.clamp_min(2.0 ** -108) / 448.0))
    return torch.exp2(e.clamp(-117, 119))


def _exact_cache(held, x=None, row0=0):
    """Values and scales of a cache that was written `held` [rows, Hkv, D] and then x at row0, from block 0 on."""
    def blocks(t, lead=0):
        n = lead + t.shape[0]
        y = torch.zeros(((n + BLOCK - 1) // BLOCK * BLOCK,) + t.shape[1:], dtype=torch.float64, device="cuda")
        y[lead:n] = t.double()
        return y
    spread = lambda s: s.repeat_interleave(BLOCK, 0)[:, :, None]
    y = blocks(held)
    s = _exact_scales(y)
    y = _nearest(y, spread(s))
    if x is None:
        return y, s
    b = row0 // BLOCK
    z = blocks(x, row0 - b * BLOCK)
    t = _exact_scales(z)
    if row0 % BLOCK:
        t[0] = torch.maximum(t[0], s[b])
        z[: row0 - b * BLOCK] = y[b * BLOCK:row0]
    return torch.cat([y[: b * BLOCK], _nearest(z, spread(t))]), torch.cat([s[:b], t])


def exact(case, seed):
    x = _inputs(case, seed)
    c = x["case"]
    if c["kind"] == "logprobs":
        N, B, V, K = c["N"], c["B"], c["V"], c["top"]
        f = lambda *s: torch.zeros(s, dtype=torch.float64, device="cuda")
        lp, ent, ids, tlp = f(N * B), f(N * B), torch.zeros((N * B, K), dtype=torch.int32, device="cuda"), f(N * B, K)
        flat, tok = x["logits"].view(N * B, V), x["tokens"].view(-1)
        for r in range(N * B):
            if x["mask"] is not None and not bool(x["mask"].view(-1)[r]):
                continue
            z = flat[r].double() / c["temperature"]
            logp = z - torch.logsumexp(z, 0)
            lp[r] = logp[tok[r].long()]
            ent[r] = torch.special.entr(torch.exp(logp)).sum()
            if K:
                i = torch.sort(z, descending=True, stable=True).indices[:K]
                ids[r], tlp[r] = i.to(torch.int32), logp[i]
        return lp.view(N, B), ent.view(N, B), ids.view(N, B, K), tlp.view(N, B, K)
    Hkv, D = c["Hkv"], c["D"]
    if c["kind"] in ("write", "read"):
        first = c["row0"] // BLOCK * BLOCK if c["kind"] == "write" else c["row0"]
        last = c["row0"] + c["rows"]
        values, scales = [], []
        for j, name in enumerate(("k", "v")):
            y, s = _exact_cache(x["held"][j], x[name], c["row0"]) if c["kind"] == "write" else _exact_cache(x["held"][j])
            all_scales = torch.ones((Hkv, _capacity(c) // BLOCK), dtype=torch.float64, device="cuda")
            all_scales[:, : s.shape[0]] = s.T
            values.append(y[first:last].contiguous())
            scales.append(all_scales)
        return (*values, *scales) if c["kind"] == "write" else tuple(values)
    N, B, L, Hq, E, P = (c[k] for k in ("N", "B", "L", "Hq", "E", "problems"))
    G = Hq // Hkv
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda")
    for p in range(P):
        of = (lambda t: t[p]) if P > 1 else (lambda t: t)
        q, o = of(x["q"]).double(), of(out)
        pk, pv = (_exact_cache(t)[0][:L] for t in x["rows"][p])
        for n in range(N):
            k = [pk, of(x["block_k"])[n].double()]
            v = [pv, of(x["block_v"])[n].double()]
            if E:
                k.insert(1, of(x["ext_k"])[n, :E].double())
                v.insert(1, of(x["ext_v"])[n, :E].double())
            k, v = torch.cat(k), torch.cat(v)
            for h in range(Hkv):
                s = (q[n, :, h * G:(h + 1) * G].reshape(B * G, D) @ k[:, h].T.contiguous()) / math.sqrt(D)
                if c["causal"]:
                    b = torch.arange(B, device="cuda")
                    s[:, L + E:] += torch.where(b[None, :] > b.repeat_interleave(G)[:, None], -math.inf, 0.0)
                w = torch.softmax(s, -1)
                o[n, :, h * G:(h + 1) * G] = (w @ v[:, h].contiguous()).view(B, G, D)
    if x["positions"] is not None:
        drop = torch.ones(N * B, dtype=torch.bool, device="cuda")
        drop[x["positions"].long()] = False
        out.view(N * B, Hq, D)[drop] = 0.0
    return out
