"""Oracle of caches in 4 bits, rows of new tokens and step tables (numpy, fp64, plain loops over what is discrete).

Test infrastructure only, like the rest of this package.  The layout of a tile is written here from its description in
the C header and shares nothing with the kernels.
"""
from __future__ import annotations

import numpy as np

SIZES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def tile_bytes(d: int) -> int:
    return 16 * d + 64 * (d // 32)


def encode(x):
    """Codes (0..15) and fp16 scales of rows [..., d]: the nearest magnitude, of two equally near the even code."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(x.shape[:-1] + (-1, 32))
    scale = np.minimum(np.abs(blocks).max(-1) / 6.0, 65504.0).astype(np.float16)
    scale[scale == 10920] = 10912                            # six times 10,920 is more than fp16 holds
    s = scale.astype(np.float64)[..., None]
    y = np.where(s > 0, np.abs(blocks) / np.where(s > 0, s, 1.0), 0.0)
    away = np.abs(y[..., None] - SIZES)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])               # even codes first: a tie goes to them
    code = order[np.argmin(away[..., order], -1)]
    code = np.where((blocks < 0) & (code > 0), code + 8, code)
    return code.reshape(x.shape), scale


def values(code, scale):
    """The values of codes [..., d] with scales [..., d / 32]."""
    v = SIZES[code & 7] * np.where(code > 7, -1.0, 1.0)
    return (v.reshape(v.shape[:-1] + (-1, 32)) * scale.astype(np.float64)[..., None]).reshape(v.shape)


def _k_byte(d, row, dim):
    return row * (d // 2) + dim % 32 // 8 * (d // 8) + 4 * (dim // 32) + dim % 8 // 2


def _v_byte(d, row, dim):
    byte = dim // 2
    if d == 128 and row >= 8:
        byte ^= 32
    return 8 * d + row * (d // 2) + byte


def _k_scale(d, row, block):
    return 16 * d + 2 * (row * (d // 32) + block)


def _v_scale(d, row, block):
    return 16 * d + 32 * (d // 32) + 2 * (16 * block + 4 * (row // 4) + ((row % 4) ^ (row // 4)))


def _index(d, which):
    """Byte of every (row, dim) and of every (row, block) of a tile."""
    byte, scale = (_k_byte, _k_scale) if which == "k" else (_v_byte, _v_scale)
    return (np.array([[byte(d, r, x) for x in range(d)] for r in range(16)]),
            np.array([[scale(d, r, b) for b in range(d // 32)] for r in range(16)]))


def put_row(tile, which, row, code, scale):
    """Writes one token's codes [d] and scales [d / 32] into a tile (uint8 [tile_bytes], modified)."""
    d = code.shape[0]
    bytes_at, scales_at = _index(d, which)
    pairs = code[0::2] | (code[1::2] << 4)
    tile[bytes_at[row, 0::2]] = pairs.astype(np.uint8)
    raw = np.ascontiguousarray(scale.astype(np.float16)).view(np.uint8).reshape(-1, 2)
    tile[scales_at[row]] = raw[:, 0]
    tile[scales_at[row] + 1] = raw[:, 1]


def pool_of(k, v, page_size, fill=0):
    """A packed pool [pages, heads, bytes] of K and V [pages, page_size, heads, d]."""
    pages, _, heads, d = k.shape
    t = page_size // 16
    out = np.full((pages, heads, t, tile_bytes(d)), fill, dtype=np.uint8)
    for which, x in (("k", k), ("v", v)):
        code, scale = encode(x)
        bytes_at, scales_at = _index(d, which)
        c = code.reshape(pages, t, 16, heads, d).transpose(0, 3, 1, 2, 4)
        s = scale.reshape(pages, t, 16, heads, d // 32).transpose(0, 3, 1, 2, 4)
        out[..., bytes_at[:, 0::2]] = (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)
        raw = np.ascontiguousarray(s).view(np.uint8).reshape(s.shape + (2,))
        out[..., scales_at] = raw[..., 0]
        out[..., scales_at + 1] = raw[..., 1]
    return out.reshape(pages, heads, -1)


def pool_values(pool, d, page_size):
    """K and V [pages, page_size, heads, d] in fp64 of a packed pool [pages, heads, bytes]."""
    pages, heads = pool.shape[:2]
    t = page_size // 16
    tiles = pool.reshape(pages, heads, t, tile_bytes(d))
    out = []
    for which in ("k", "v"):
        bytes_at, scales_at = _index(d, which)
        byte = tiles[..., bytes_at]
        code = np.where(np.arange(d) % 2 == 0, byte & 15, byte >> 4).astype(np.int64)
        raw = np.stack([tiles[..., scales_at], tiles[..., scales_at + 1]], -1)
        scale = np.ascontiguousarray(raw).view(np.float16)[..., 0]
        out.append(values(code, scale).transpose(0, 2, 3, 1, 4).reshape(pages, page_size, heads, d))
    return out


def attend(q, k, v, table, lens, page_size, window=0, sinks=0, scale=None):
    """One query per sequence: q [b, hq, d]; K and V values of the pool.  Returns out, lse, and per output the sum of weight
    * |value| and per row the largest sum of |q k| scaled: what error bounds are counted from."""
    b, hq, d = q.shape
    hkv = k.shape[2]
    g = hq // hkv
    scale = np.float64(np.float32(1.0) / np.sqrt(np.float32(d))) if scale is None else np.float64(np.float32(scale))
    out, lse = np.zeros((b, hq, d)), np.full((b, hq), -np.inf)
    mass, size = np.zeros((b, hq, d)), np.zeros((b, hq))
    for i in range(b):
        at = np.arange(lens[i])
        if window:
            at = at[(at >= lens[i] - window) | (at < sinks)]
        if len(at) == 0:
            continue
        page = table[i][at // page_size]
        for h in range(hq):
            kk, vv = k[page, at % page_size, h // g], v[page, at % page_size, h // g]
            x = scale * (kk @ q[i, h])
            size[i, h] = (scale * (np.abs(kk) @ np.abs(q[i, h]))).max()
            m = x.max()
            p = np.exp(x - m)
            lse[i, h] = m + np.log(p.sum())
            p = p / p.sum()
            out[i, h] = p @ vv
            mass[i, h] = p @ np.abs(vv)
    return out, lse, mass, size


def rows(x, weight, eps, turn, interleaved):
    """Heads [n, h, d] in fp64: normed with weight ([d] or [h, d] or None), rotated by turn [n, rotary] or None."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    if turn is not None:
        half = turn.shape[1] // 2
        c, s = turn[:, None, :half], turn[:, None, half:]
        first = np.arange(half) * 2 if interleaved else np.arange(half)
        second = first + 1 if interleaved else first + half
        a, b = x[..., first].copy(), x[..., second].copy()
        x[..., first], x[..., second] = a * c - b * s, b * c + a * s
    return x


OK, INVALID, SMALL, STALE, BAD_PAGE, NO_PAGES = 0, -1, -3, -4, -6, -8


def step_tables(lens, gains, table, free, count, capacity, page_size, num_pages, max_rows):
    """The step as the header describes it, sequence by sequence.  `table` and `free` are modified copies in the result."""
    lens, gains, table, free = list(lens), list(gains), [list(r) for r in table], list(free)
    width, status = (len(table[0]) if table else 0), OK
    n = len(lens)
    out = list(lens)
    if not 0 <= count <= capacity:
        rest = [-1] * max_rows
        return {"lens": out, "count": count, "free": free, "table": table, "row_starts": [0] * (n + 1),
                "page_starts": [0] * (n + 1), "slots": rest, "positions": rest, "row_seq": rest, "status": STALE}
    pages = lambda t: -(-t // page_size)
    good = []
    for b in range(n):
        new = max(0, lens[b] + gains[b])
        good.append(0 <= lens[b] <= width * page_size and new <= width * page_size)
        if not good[b]:
            status = min(status, STALE)
    full = count
    back_sum = 0
    for b in range(n):
        if not good[b] or gains[b] >= 0:
            continue
        new = max(0, lens[b] + gains[b])
        ids = table[b][pages(new):pages(lens[b])]
        back_sum += len(ids)
        if ids and count + back_sum > capacity:
            status = min(status, NO_PAGES)
            continue
        free[full:full + len(ids)] = ids
        full += len(ids)
        out[b] = new
    row_starts, page_starts, slots, positions, seqs = [0], [0], [], [], []
    lack_sum = row_sum = taken = 0
    for b in range(n):
        served = False
        if good[b] and gains[b] > 0:
            lack = pages(lens[b] + gains[b]) - pages(lens[b])
            lack_sum, row_sum = lack_sum + lack, row_sum + gains[b]
            served = True
            if lack and lack_sum > full:
                served, status = False, min(status, NO_PAGES)
            if row_sum > max_rows:
                served, status = False, min(status, SMALL)
        if served:
            for i in range(pages(lens[b]), pages(lens[b] + gains[b])):
                table[b][i] = free[full - 1 - taken]
                taken += 1
            out[b] = lens[b] + gains[b]
            for p in range(lens[b], out[b]):
                page = table[b][p // page_size]
                if not 0 <= page < num_pages:
                    status = min(status, BAD_PAGE)
                slots.append(page * page_size + p % page_size if 0 <= page < num_pages else -1)
                positions.append(p)
                seqs.append(b)
        row_starts.append(len(slots))
        page_starts.append(taken)
    rest = [-1] * (max_rows - len(slots))
    return {"lens": out, "count": full - taken, "free": free, "table": table, "row_starts": row_starts,
            "page_starts": page_starts, "slots": slots + rest, "positions": positions + rest, "row_seq": seqs + rest,
            "status": status}
