"""How fdd_paged_attn deals a call's keys to workgroups, in plain Python (test infrastructure)."""
import collections

XCDS, CUS, MIN_TILES = 8, 256, 2

Item = collections.namedtuple("Item", "n kh mt piece pieces t_begin t_end whole")


def ceil(a, b):
    return -(-a // b)


def plan(N, B, Hq, Hkv, bf16, capacity, max_len=0):
    """(wavefronts of a workgroup, those that can have rows, keys of a tile, pieces aimed at, pieces at most, whether a request may have more than one)"""
    rows = B * (Hq // Hkv)
    waves = 4 if rows <= 128 or (rows <= 256 and N * Hkv <= 32) or not bf16 else 8
    used, kt, W = min(waves, ceil(rows, 32)), 64 if bf16 else 32, CUS if waves == 8 else 2 * CUS
    longest = min(max_len, capacity) if max_len else capacity
    partials = ceil(longest, kt) + ceil(B, kt) > MIN_TILES
    return waves, used, kt, W, N * Hkv * ceil(rows, waves * 32) + (W if partials else 0), partials


def requests(lens, counts, G, waves, kt):
    """(M-tiles of a KV head, tiles of keys) of every request"""
    return [(ceil(c * G, waves * 32), ceil(L, kt) + ceil(c, kt)) for L, c in zip(lens, counts)]


def tiles_of_a_piece(reqs, Hkv, W):
    return max(MIN_TILES, ceil(sum(m * t for m, t in reqs) * Hkv, W))


def items(lens, counts, B, Hq, Hkv, bf16, capacity, max_len=0, causal=False):
    """What workgroup 0, 1, .. has; `whole`: the steps that request whole tiles of the cache only."""
    G = Hq // Hkv
    waves, _, kt, W, _, _ = plan(len(lens), B, Hq, Hkv, bf16, capacity, max_len)
    lens = [min(L, capacity, max_len or capacity) for L in lens]
    reqs = requests(lens, counts, G, waves, kt)
    per = tiles_of_a_piece(reqs, Hkv, W)
    slots = 4 if waves == 8 else 2
    out = []
    for n, (mtiles, tiles) in enumerate(reqs):
        pieces = ceil(tiles, per)
        for i in range(Hkv * mtiles * pieces):
            group, at = divmod(i, XCDS * mtiles) if mtiles else (0, 0)
            wide = min(XCDS, Hkv * pieces - group * XCDS)
            kh, piece = divmod(group * XCDS + at % wide, pieces)
            each, more = divmod(tiles, pieces)
            t0 = each * piece + min(piece, more)
            t1 = t0 + each + (piece < more)
            if causal:
                mrows = ceil(ceil(counts[n] * G, 32), mtiles) * 32
                last = (min((at // wide + 1) * mrows, counts[n] * G) - 1) // G
                t1 = min(t1, ceil(lens[n], kt) + last // kt + 1)
            out.append(Item(n, kh, at // wide, piece, pieces, t0, t1, max(0, min(t1, lens[n] // kt) - t0 - slots) // 2 * 2))
    return out


def joined_at(lens, counts, B, Hq, Hkv, bf16, capacity, n, kh, mt, piece, max_len=0):
    """The item that the merge takes a piece's partial results from."""
    waves, _, kt, W, _, _ = plan(len(lens), B, Hq, Hkv, bf16, capacity, max_len)
    lens = [min(L, capacity, max_len or capacity) for L in lens]
    reqs = requests(lens, counts, Hq // Hkv, waves, kt)
    per = tiles_of_a_piece(reqs, Hkv, W)
    base = sum(Hkv * m * ceil(t, per) for m, t in reqs[:n])
    pieces = ceil(reqs[n][1], per)
    head_piece = kh * pieces + piece
    group = head_piece // XCDS
    wide = min(XCDS, Hkv * pieces - group * XCDS)
    return base + group * XCDS * reqs[n][0] + mt * wide + head_piece - group * XCDS
