"""ctypes binding of the operators on a paged cache and on trees of drafted tokens (see include/fdd.h).

Argument marshalling only, as in ``binding``.  All tensors of a call live on the current device.
"""
from __future__ import annotations

import ctypes as C
from typing import Any, NamedTuple

from . import binding as _b
from .binding import FDD_ATTN_CAUSAL_BLOCK, _check, _check_out, _check_workspace, _dev, _device_and_stream, _dtype_code, _maker, _on_current_device, \
    _set_workspace, load_library

FDD_ROPE_INVERSE = 1
FDD_TREE_MAX = 1024
_SCALINGS = {None: 0, "linear": 1, "base": 2, "parts": 3}


class RopeScaling(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("scaling", C.c_int32), ("base", C.c_double), ("stretch", C.c_double), ("original", C.c_double)]


class RopeTableStruct(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("magnitude", C.c_float), ("reserved", C.c_int32)]


class RopeParams(C.Structure):
    _fields_ = [("rows", C.c_int32), ("Hq", C.c_int32), ("Hk", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32), ("flags", C.c_int32),
                ("table", RopeTableStruct), ("positions", C.c_void_p), ("q", C.c_void_p), ("q_out", C.c_void_p), ("k", C.c_void_p), ("k_out", C.c_void_p),
                ("q_stride", C.c_int64), ("q_out_stride", C.c_int64), ("k_stride", C.c_int64), ("k_out_stride", C.c_int64), ("stream", C.c_void_p)]


class PagedCacheStruct(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_table", C.c_void_p), ("lens", C.c_void_p), ("N", C.c_int32), ("pages", C.c_int32),
                ("page_size", C.c_int32), ("max_pages", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class AppendParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("reserved", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_stride", C.c_int64), ("v_stride", C.c_int64),
                ("rope", C.c_void_p), ("positions", C.c_void_p), ("rows", C.c_void_p), ("n_rows", C.c_void_p), ("stream", C.c_void_p)]


class TreeMaskParams(C.Structure):
    _fields_ = [("N", C.c_int32), ("B", C.c_int32), ("parents", C.c_void_p), ("parents_stride", C.c_int64), ("lens", C.c_void_p),
                ("n_tokens", C.c_void_p), ("mask", C.c_void_p), ("positions", C.c_void_p), ("stream", C.c_void_p)]


class PagedAttnParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("flags", C.c_int32), ("max_len", C.c_int32), ("scale", C.c_float), ("reserved", C.c_int32),
                ("q", C.c_void_p), ("block_k", C.c_void_p), ("block_v", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64),
                ("v_stride", C.c_int64), ("mask", C.c_void_p), ("mask_stride", C.c_int64), ("n_tokens", C.c_void_p), ("out", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class TreeVerifyParams(C.Structure):
    _fields_ = [("N", C.c_int32), ("B", C.c_int32), ("V", C.c_int64), ("dtype", C.c_int32), ("temperature", C.c_float),
                ("draft_temperature", C.c_float), ("reserved", C.c_int32), ("logits", C.c_void_p), ("draft_logits", C.c_void_p),
                ("tokens", C.c_void_p), ("parents", C.c_void_p), ("parents_stride", C.c_int64), ("uniforms", C.c_void_p), ("n_tokens", C.c_void_p),
                ("path", C.c_void_p), ("n_path", C.c_void_p), ("emitted", C.c_void_p), ("chances", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class AppendCall(C.Structure):
    _fields_ = [("cache", PagedCacheStruct), ("p", AppendParams), ("table", RopeTableStruct)]


class PagedAttnCall(C.Structure):
    _fields_ = [("cache", PagedCacheStruct), ("p", PagedAttnParams)]


_BYTES = dict(rope_bytes=RopeParams, append_bytes=AppendCall, tree_mask_bytes=TreeMaskParams, paged_attn_bytes=PagedAttnCall, tree_verify_bytes=TreeVerifyParams)
_APPEND_AT, _ATTN_AT = AppendCall.p.offset, PagedAttnCall.p.offset
_fits = {}      # whether a module's structs are these


def _marshal():
    """The native argument marshalling, or None where it was not built, or from another header."""
    m = _b._marshal
    if m is None:
        return None
    if m not in _fits:
        _fits[m] = all(getattr(m, name, None) == C.sizeof(t) for name, t in _BYTES.items())
    return m if _fits[m] else None


class PagedCache(NamedTuple):
    """K and V of N requests in pages: ``k``, ``v`` [pages,Hkv,page_size,D], ``page_table`` int32 [N,max_pages] and ``lens`` int32 [N],
    the rows that each request holds.  Both lists are read when a call runs."""
    k: Any
    v: Any
    page_table: Any
    lens: Any


class RopeTable(NamedTuple):
    """Frequencies of the rotation: ``turns`` int64 [rot_dim/2], parts of a turn in 2^-64 (the bits of an unsigned number)."""
    turns: Any
    interleaved: bool = False
    magnitude: float = 1.0


def _typed(t, dtype, shape, name):
    if t is None:
        return None
    if t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise TypeError(f"{name} must be {dtype} {list(shape)}")
    return _dev(t, name)


def _tokens(t, name, shape):
    """Address of an array [N,B,heads,D] and the stride of its tokens, which may lie apart (a part of a fused projection)."""
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must live in GPU memory")
    N, B, H, D = shape
    s = t.stride()
    # (the stride of a dimension of one entry means nothing)
    if (D > 1 and s[3] != 1) or (H > 1 and s[2] != D):
        raise ValueError(f"the heads and channels of a token of {name} must be contiguous")
    step = s[1] if B > 1 else s[0] if N > 1 else H * D
    if N > 1 and B > 1 and s[0] != B * step:
        raise ValueError(f"tokens of {name} must be evenly spaced")
    if step < H * D:
        raise ValueError(f"tokens of {name} must not overlap")
    return t.data_ptr(), step


def _tree(t, name, N, tail, dtype):
    """Address of an array for each request, or for all of them, and the entries from one request's to the next."""
    if t is None:
        return None, 0
    shape = tuple(t.shape)
    if t.dtype != dtype or shape not in (tuple(tail), (N,) + tuple(tail)):
        raise TypeError(f"{name} must be {dtype} {[N] + list(tail)}, or {list(tail)} for all requests")
    n = 1
    for x in tail:
        n *= x
    return _dev(t, name), n if len(shape) == len(tail) + 1 else 0


def fdd_rope_table(rot_dim, base=10000.0, interleaved=False, scaling=None, stretch=1.0, original=None, device="cuda") -> RopeTable:
    """Frequencies base^(-2i / rot_dim) for ``rot_dim`` rotated channels.  ``scaling`` for contexts longer than trained: "linear",
    "base" or "parts" (which needs the ``original`` length), all by ``stretch``.  ``interleaved``: pairs are neighbours (2i, 2i+1)
    instead of (i, i + rot_dim/2)."""
    lib = load_library()
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {list(_SCALINGS)}")
    if scaling == "parts" and original is None:
        raise ValueError('scaling "parts" needs the original length')
    rot_dim = int(rot_dim)
    p = RopeScaling(rot_dim, _SCALINGS[scaling], float(base), float(stretch), 1.0 if original is None else float(original))
    turns = (C.c_uint64 * max(1, rot_dim // 2))()
    magnitude = C.c_float()
    _check(lib.fdd_rope_turns(C.byref(p), turns, C.byref(magnitude)))
    t = _b.torch.frombuffer(bytearray(turns), dtype=_b.torch.int64).to(device)
    return RopeTable(t, bool(interleaved), magnitude.value)


def _table_struct(table, D):
    turns, interleaved, magnitude = table
    if turns.dtype != _b.torch.int64 or turns.dim() != 1:
        raise TypeError("turns must be a 1-D int64 tensor")
    _on_current_device(turns)
    s = RopeTableStruct()
    s.turns, s.rot_dim, s.interleaved, s.magnitude = _dev(turns, "turns"), 2 * turns.numel(), 1 if interleaved else 0, float(magnitude)
    return s


def _rope_array(t, name, lead):
    """Address of [..,heads,D] and the stride of its rows."""
    if t.dim() < 2 or tuple(t.shape[:-2]) != tuple(lead):
        raise ValueError(f"{name} must be {list(lead)} + [heads,D]")
    if not t.is_cuda:
        raise ValueError(f"{name} must live in GPU memory")
    H, D = t.shape[-2:]
    s = t.stride()
    if t.numel() and ((D > 1 and s[-1] != 1) or (H > 1 and s[-2] != D)):
        raise ValueError(f"the heads and channels of a row of {name} must be contiguous")
    step, rows = 0, 1
    for n, st in zip(reversed(lead), reversed(s[:-2])):      # rows must be evenly spaced over all leading dimensions
        if n > 1 and t.numel():
            if rows > 1 and st != step * rows:
                raise ValueError(f"rows of {name} must be evenly spaced")
            step = step if rows > 1 else st
            rows *= n
    if rows > 1 and step < H * D:
        raise ValueError(f"rows of {name} must not overlap")
    return t.data_ptr(), step


def fdd_rope(q, positions, table, k=None, out=None, k_out=None, inverse=False, stream=None):
    """Rotary positions: q [..,Hq,D] and, if given, k [..,Hk,D] rotated at ``positions`` (int32 [..]) by the frequencies of ``table``.
    Rows may lie apart; ``out`` may be q (in place), ``k_out`` k.  ``inverse`` turns back, by the same magnitude: the gradient.
    Returns the rotated q, or (q, k)."""
    lib = load_library()
    dev, handle = _device_and_stream(stream)
    if k is None and k_out is not None:
        raise ValueError("k_out needs k")
    if out is None or (k is not None and k_out is None):
        empty = lambda x: (_b.torch.empty if stream is None else _maker(stream, x.device, _b.torch.empty))(tuple(x.shape), dtype=x.dtype, device=x.device)
        out = empty(q) if out is None else out
        k_out = empty(k) if k is not None and k_out is None else k_out
    p = RopeParams()
    m = _marshal()
    if m is None or not m.rope(C.addressof(p), q, positions, table, k, out, k_out, inverse, dev):
        p = _rope_params(q, positions, table, k, out, k_out, inverse)
    p.stream = handle
    if p.rows:
        _check(lib.fdd_rope(C.addressof(p)))
    return out if k is None else (out, k_out)


def _rope_params(q, positions, table, k, out, k_out, inverse):
    torch = _b.torch
    lead = tuple(q.shape[:-2])
    if positions.dtype != torch.int32 or tuple(positions.shape) != lead:
        raise TypeError(f"positions must be torch.int32 {list(lead)}")
    for x, o, name in ((q, out, "q"), (k, k_out, "k")):
        if x is not None and (o.shape != x.shape or o.dtype != x.dtype):
            raise ValueError(f"the output of {name} must have its shape and type")
    if k is not None and (k.dtype != q.dtype or k.shape[-1] != q.shape[-1]):
        raise TypeError("q and k must share element type and head size")
    _on_current_device(q, k, positions, out, k_out)
    p = RopeParams()
    rows = 1
    for n in lead:
        rows *= n
    p.rows, p.Hq, p.D, p.dtype, p.flags = rows, q.shape[-2], q.shape[-1], _dtype_code(q), FDD_ROPE_INVERSE if inverse else 0
    p.table = _table_struct(table, p.D)
    p.positions = _dev(positions, "positions")
    p.q, p.q_stride = _rope_array(q, "q", lead)
    p.q_out, p.q_out_stride = _rope_array(out, "out", lead)
    if k is not None:
        p.Hk = k.shape[-2]
        p.k, p.k_stride = _rope_array(k, "k", lead)
        p.k_out, p.k_out_stride = _rope_array(k_out, "k_out", lead)
    return p


def fdd_paged_cache(N, pages, page_size, max_pages, Hkv, D, dtype=None, device="cuda") -> PagedCache:
    """A cache of N requests without rows, and without pages: ``page_table`` is the caller's to fill."""
    load_library()
    torch = _b.torch
    dtype = torch.bfloat16 if dtype is None else dtype
    pool = [torch.empty((pages, Hkv, page_size, D), dtype=dtype, device=device) for _ in range(2)]
    return PagedCache(*pool, torch.full((N, max_pages), -1, dtype=torch.int32, device=device), torch.zeros((N,), dtype=torch.int32, device=device))


def _cache_struct(cache):
    k, v, table, lens = cache
    torch = _b.torch
    if k.dim() != 4 or v.shape != k.shape:
        raise ValueError("a paged cache is k, v [pages,Hkv,page_size,D], page_table [N,max_pages] and lens [N]")
    if v.dtype != k.dtype:
        raise TypeError("k and v of a cache must share one element type")
    if table.dtype != torch.int32 or table.dim() != 2 or lens.dtype != torch.int32 or tuple(lens.shape) != (table.shape[0],):
        raise TypeError("page_table must be torch.int32 [N,max_pages] and lens torch.int32 [N]")
    _on_current_device(*cache)
    c = PagedCacheStruct(_dev(k, "cache k"), _dev(v, "cache v"), _dev(table, "page_table"), _dev(lens, "lens"))
    c.N, c.max_pages = table.shape
    c.pages, c.Hkv, c.page_size, c.D = k.shape
    c.dtype = _dtype_code(k)
    return c


def fdd_paged_append(k, v, cache, table=None, positions=None, rows=None, n_rows=None, stream=None):
    """Rows of k, v [N,B,Hkv,D] join the pages of ``cache`` (in place) behind the ``lens`` rows that each request holds; k is rotated
    by ``table`` on the way, if given, at ``positions`` (int32 [N,B]) or where the row comes to lie.  ``rows`` (int32 [N,B]) names the source row of
    every new one, ``n_rows`` (int32 [N]) how many there are: ``path`` and ``n_path`` of fdd_tree_verify.  ``lens`` stays as it is: add
    ``n_rows`` to it once every layer's call has been made."""
    lib = load_library()
    dev, handle = _device_and_stream(stream)
    call = AppendCall()
    m = _marshal()
    if m is None or not m.append(C.addressof(call), k, v, cache, table, positions, rows, n_rows, dev):
        call = AppendCall()
        _append_params(call, k, v, cache, table, positions, rows, n_rows)
    call.p.stream = handle
    _check(lib.fdd_paged_append(C.addressof(call), C.addressof(call) + _APPEND_AT))


def _append_params(call, k, v, cache, table, positions, rows, n_rows):
    torch = _b.torch
    c = call.cache = _cache_struct(cache)
    if k.dim() != 4:
        raise ValueError("k and v must be [N,B,Hkv,D]")
    B = k.shape[1]
    if k.dtype != v.dtype or _dtype_code(k) != c.dtype:
        raise TypeError("k and v must have the cache's element type")
    _on_current_device(k, v, positions, rows, n_rows)
    p = call.p
    p.B = B
    p.k, p.k_stride = _tokens(k, "k", (c.N, B, c.Hkv, c.D))
    p.v, p.v_stride = _tokens(v, "v", (c.N, B, c.Hkv, c.D))
    if table is not None:
        call.table = _table_struct(table, c.D)
        p.rope = C.addressof(call.table)
    p.positions = _typed(positions, torch.int32, (c.N, B), "positions")
    p.rows = _typed(rows, torch.int32, (c.N, B), "rows")
    p.n_rows = _typed(n_rows, torch.int32, (c.N,), "n_rows")


def fdd_tree_mask(parents, lens=None, n_tokens=None, mask=None, positions=None, N=None, stream=None):
    """What the tokens of drafted trees see and where they stand.  ``parents`` int32 [N,B], or [B] for all requests (with ``lens``,
    ``n_tokens`` or ``N`` to say how many).  Returns (mask int64 [N,B,ceil(B/64)], the bits of fdd_paged_attn's ``mask``, positions int32 [N,B])."""
    lib = load_library()
    dev, handle = _device_and_stream(stream)
    p = TreeMaskParams()
    m = _marshal()
    if mask is not None and positions is not None and N is None and m is not None and m.tree_mask(C.addressof(p), parents, lens, n_tokens, mask, positions, dev):
        p.stream = handle
        _check(lib.fdd_tree_mask(C.addressof(p)))
        return mask, positions
    torch = _b.torch
    if parents.dim() not in (1, 2):
        raise TypeError("parents must be torch.int32 [N,B] or [B]")
    B = parents.shape[-1]
    if N is None:
        N = next((t.shape[0] for t in ((parents if parents.dim() == 2 else None), lens, n_tokens, mask, positions) if t is not None), 1)
    N = int(N)
    words = (B + 63) // 64
    new = torch.empty if stream is None else _maker(stream, parents.device, torch.empty)
    if mask is None:
        mask = new((N, B, words), dtype=torch.int64, device=parents.device)
    if positions is None:
        positions = new((N, B), dtype=torch.int32, device=parents.device)
    _on_current_device(parents, lens, n_tokens, mask, positions)
    p = TreeMaskParams()
    p.N, p.B = N, B
    p.parents, p.parents_stride = _tree(parents, "parents", N, (B,), torch.int32)
    p.lens, p.n_tokens = _typed(lens, torch.int32, (N,), "lens"), _typed(n_tokens, torch.int32, (N,), "n_tokens")
    p.mask, p.positions = _typed(mask, torch.int64, (N, B, words), "mask"), _typed(positions, torch.int32, (N, B), "positions")
    p.stream = handle
    _check(lib.fdd_tree_mask(C.addressof(p)))
    return mask, positions


def _paged_attn_params(q, cache, block_k, block_v, mask, n_tokens, out, scale, causal_block, max_len):
    torch = _b.torch
    c = _cache_struct(cache)
    if q.dim() != 4:
        raise ValueError("q must be [N,B,Hq,D]")
    N, B, Hq, D = q.shape
    if N != c.N or D != c.D:
        raise ValueError("q must have the cache's N and D")
    if q.dtype != block_k.dtype or q.dtype != block_v.dtype or _dtype_code(q) != c.dtype:
        raise TypeError("q, block_k and block_v must have the cache's element type")
    _check_out(out, q)
    _on_current_device(q, block_k, block_v, mask, n_tokens, out)
    p = PagedAttnParams()
    p.B, p.Hq, p.flags, p.max_len = B, Hq, FDD_ATTN_CAUSAL_BLOCK if causal_block else 0, int(max_len)
    p.scale = 0.0 if scale is None else float(scale)
    p.q, p.q_stride = _tokens(q, "q", (N, B, Hq, D))
    p.block_k, p.k_stride = _tokens(block_k, "block_k", (N, B, c.Hkv, D))
    p.block_v, p.v_stride = _tokens(block_v, "block_v", (N, B, c.Hkv, D))
    p.mask, p.mask_stride = _tree(mask, "mask", N, (B, (B + 63) // 64), torch.int64)
    p.n_tokens = _typed(n_tokens, torch.int32, (N,), "n_tokens")
    p.out = _dev(out, "out")
    return p, c


def fdd_paged_attn_workspace(q, cache, block_k, block_v, max_len=0) -> int:
    """Workspace bytes of the fdd_paged_attn call with these arguments."""
    lib = load_library()
    p, c = _paged_attn_params(q, cache, block_k, block_v, None, None, None, None, False, max_len)
    return lib.fdd_paged_attn_workspace(C.addressof(c), C.addressof(p))


def fdd_paged_attn(q, cache, block_k, block_v, mask=None, n_tokens=None, causal_block=False, max_len=0, scale=None, out=None, workspace=None,
                   stream=None):
    """Attention of every request's new tokens, q [N,B,Hq,D], over the rows of its paged cache and over block_k, block_v [N,B,Hkv,D], the
    new tokens' own (see include/fdd.h).  ``mask`` int64 [N,B,ceil(B/64)] (or without N, for all requests): what a token sees of the block, as
    fdd_tree_mask makes it; else all of it, or with ``causal_block`` what is not behind it.  ``n_tokens`` int32 [N]: how many of the B tokens are
    there; rows of ``out`` behind them stay as they were (0 in an ``out`` that is allocated here).  ``max_len``: no request holds more rows."""
    lib = load_library()
    dev, handle = _device_and_stream(stream)
    torch = _b.torch
    if out is None:
        make = torch.empty if n_tokens is None else torch.zeros
        out = (make if stream is None else _maker(stream, q.device, make))(tuple(q.shape), dtype=q.dtype, device=q.device)
    call = PagedAttnCall()
    m = _marshal()
    if m is None or not m.paged_attn(C.addressof(call), q, cache, block_k, block_v, mask, n_tokens, causal_block, max_len, scale, out, dev):
        call.p, call.cache = _paged_attn_params(q, cache, block_k, block_v, mask, n_tokens, out, scale, causal_block, max_len)
    _check_workspace(workspace, dev)
    at = C.addressof(call)
    p = call.p
    ws = _set_workspace(p, workspace, lambda _: lib.fdd_paged_attn_workspace(at, at + _ATTN_AT), q.device, stream)  # noqa: F841
    p.stream = handle
    _check(lib.fdd_paged_attn(at, at + _ATTN_AT))
    return out


def _verify_params(logits, draft_logits, temperature, draft_temperature):
    if logits.dim() != 3:
        raise ValueError("logits must be [N,B,V]")
    p = TreeVerifyParams()
    p.N, p.B, p.V = logits.shape
    p.dtype, p.temperature, p.draft_temperature = _dtype_code(logits), float(temperature), float(draft_temperature)
    if draft_logits is not None:
        if draft_logits.shape != logits.shape or draft_logits.dtype != logits.dtype:
            raise TypeError("draft_logits must have the shape and type of logits")
        p.draft_logits = _dev(draft_logits, "draft_logits")
    return p


def fdd_tree_verify_workspace(logits, draft_logits=None) -> int:
    """Workspace bytes of fdd_tree_verify calls with these arguments, at any temperature."""
    lib = load_library()
    p = _verify_params(logits, draft_logits, 1.0, 1.0)
    return lib.fdd_tree_verify_workspace(C.addressof(p))


def fdd_tree_verify(logits, tokens, uniforms=None, parents=None, draft_logits=None, n_tokens=None, temperature=1.0, draft_temperature=1.0, path=None,
                    n_path=None, emitted=None, chances=None, workspace=None, stream=None):
    """Which drafted tokens stand, from the target's ``logits`` [N,B,V] and random numbers ``uniforms`` (float32 [N,B,2] in [0,1)), and the
    token behind them (see include/fdd.h).  ``tokens`` int32 [N,B], token 0 the last certain one; ``parents`` int32 [N,B] or [B], None for a
    chain; ``draft_logits`` of a chain whose tokens were drawn from them.  ``temperature`` 0: greedy.

    Returns (path int32 [N,B], n_path int32 [N], emitted int32 [N,B], chances float32 [N,B])."""
    lib = load_library()
    dev, handle = _device_and_stream(stream)
    m = _marshal()
    p = TreeVerifyParams()
    if path is None or n_path is None or emitted is None or chances is None or m is None or not m.tree_verify(
            C.addressof(p), logits, tokens, uniforms, parents, draft_logits, n_tokens, temperature, draft_temperature, path, n_path, emitted, chances, dev):
        p, path, n_path, emitted, chances = _verify_arguments(logits, tokens, uniforms, parents, draft_logits, n_tokens, temperature, draft_temperature, path,
                                                              n_path, emitted, chances, stream)
    _check_workspace(workspace, dev)
    ws = _set_workspace(p, workspace, lambda _: lib.fdd_tree_verify_workspace(C.addressof(p)), logits.device, stream)  # noqa: F841
    p.stream = handle
    _check(lib.fdd_tree_verify(C.addressof(p)))
    return path, n_path, emitted, chances


def _verify_arguments(logits, tokens, uniforms, parents, draft_logits, n_tokens, temperature, draft_temperature, path, n_path, emitted, chances, stream):
    torch = _b.torch
    p = _verify_params(logits, draft_logits, temperature, draft_temperature)
    N, B = p.N, p.B
    new = torch.empty if stream is None else _maker(stream, logits.device, torch.empty)
    outs = []
    for t, shape, dtype in ((path, (N, B), torch.int32), (n_path, (N,), torch.int32), (emitted, (N, B), torch.int32), (chances, (N, B), torch.float32)):
        outs.append(new(shape, dtype=dtype, device=logits.device) if t is None else t)
    _on_current_device(logits, draft_logits, tokens, uniforms, parents, n_tokens, *outs)
    p.logits = _dev(logits, "logits")
    p.tokens = _typed(tokens, torch.int32, (N, B), "tokens")
    p.uniforms = _typed(uniforms, torch.float32, (N, B, 2), "uniforms")
    p.parents, p.parents_stride = _tree(parents, "parents", N, (B,), torch.int32)
    p.n_tokens = _typed(n_tokens, torch.int32, (N,), "n_tokens")
    p.path, p.n_path = _typed(outs[0], torch.int32, (N, B), "path"), _typed(outs[1], torch.int32, (N,), "n_path")
    p.emitted, p.chances = _typed(outs[2], torch.int32, (N, B), "emitted"), _typed(outs[3], torch.float32, (N, B), "chances")
    return (p, *outs)
