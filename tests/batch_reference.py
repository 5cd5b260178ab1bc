"""A batch of requests over one pool of blocks in 8 bits, plainly and in 64 bits: what the tests of these operators compare with."""
import math

import numpy as np

from tests import kv4_reference

GRID = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (x - 10) for x in range(1, 16) for m in range(8)])[:127]
VALUES = np.concatenate([GRID, [np.nan], -GRID, [np.nan]])


def exponent(most: np.ndarray) -> np.ndarray:
    """e + 127 of the smallest e in [-117, 119] with most <= 448 * 2^e."""
    m, x = np.frexp(most / 448.0)                                # (in 64 bits the quotient is 1/2 exactly where most is 448 times a power of two, and nowhere else for floats)
    e = np.where(m == 0.5, x - 1, x)
    return np.clip(np.where(most > 0, e, -117), -117, 119).astype(np.int64) + 127


def codes(y: np.ndarray) -> np.ndarray:
    """y[..] -> the bytes of the nearest values, ties to the even one, 448 for what is above, 127 for what is not finite."""
    odd = ~np.isfinite(y)
    a = np.minimum(np.abs(np.where(odd, 0.0, y)), 448.0)
    up = np.searchsorted(GRID, a)
    down = np.maximum(up - 1, 0)
    above, below = GRID[up] - a, a - GRID[down]
    c = np.where((above < below) | ((above == below) & (up % 2 == 0)), up, down)
    return np.where(odd, 127, c + 128 * np.signbit(np.where(odd, 0.0, y))).astype(np.uint8)


def slot_bytes(block, heads, d):
    return -(-(2 * block * heads * d + 2 * heads) // 16) * 16


def parts(slot: np.ndarray, block, heads, d, at=0):
    """Views of one slot's bytes: Keys' codes [heads, block, d], Values', exponents [heads, 2]."""
    c = heads * block * d
    x = slot[at:at + 2 * c + 2 * heads]
    return x[:c].reshape(heads, block, d), x[c:2 * c].reshape(heads, block, d), x[2 * c:].reshape(heads, 2)


def runs(row_slot, block, n_slots):
    """(first row, rows, slot, row of the block) of each stretch of rows that go to one block."""
    out, t = [], 0
    while t < len(row_slot):
        p = int(row_slot[t])
        n = 1
        if 0 <= p < n_slots * block:
            while t + n < len(row_slot) and p % block + n < block and int(row_slot[t + n]) == p + n:
                n += 1
            out.append((t, n, p // block, p % block))
        t += n
    return out


def write(pool: np.ndarray, k: np.ndarray, v: np.ndarray, row_slot, block: int, at: int = 0) -> np.ndarray:
    """What pool [slots, bytes] holds afterwards."""
    pool = pool.copy()
    H, d = k.shape[1:]
    for t, n, slot, r in runs(row_slot, block, pool.shape[0]):
        views = parts(pool[slot], block, H, d, at)
        for i, x in enumerate((k, v)):
            rows = x[t:t + n]
            byte = exponent(np.abs(np.where(np.isfinite(rows), rows, 0.0)).max((0, 2)))
            if r:
                old = np.clip(views[2][:, i].astype(np.int64), 10, 246)
                byte = np.maximum(byte, old)
                for h in np.nonzero(byte > old)[0]:
                    views[i][h, :r] = codes(VALUES[views[i][h, :r]] * 2.0 ** float(old[h] - byte[h]))
            views[i][:, r:r + n] = codes(rows / np.exp2(byte - 127.0)[None, :, None]).transpose(1, 0, 2)
            views[2][:, i] = byte
    return pool


def values(pool: np.ndarray, slots, n_tokens, block, H, d, at=0):
    """(k, v)[n_tokens, H, d] float64 of the blocks in `slots`; NaN for rows of a block that is nowhere."""
    out = np.full((2, n_tokens, H, d), np.nan)
    for b in range(-(-n_tokens // block)):
        if not 0 <= slots[b] < pool.shape[0]:
            continue
        rows = min(block, n_tokens - b * block)
        views = parts(pool[slots[b]], block, H, d, at)
        for i in (0, 1):
            x = VALUES[views[i]] * np.exp2(views[2][:, i].astype(np.float64) - 127.0)[:, None, None]
            out[i, b * block:b * block + rows] = x.transpose(1, 0, 2)[:rows]
    return out


def batch_map(lens, new, table, free, used, block, n_slots, n_rows):
    """(lens_out, row_start, row_pos, row_slot, info, table) as slim_batch_map leaves them."""
    R, wide = table.shape
    table = table.copy()
    taken = sum(-(-(l + n) // block) - -(-l // block) for l, n in zip(lens, new) if l >= 0 and n >= 0 and l + n <= wide * block)
    rows = sum(n for l, n in zip(lens, new) if l >= 0 and n >= 0 and l + n <= wide * block)
    err = (1 if any(l < 0 or n < 0 or l + n > wide * block for l, n in zip(lens, new)) else 0) | (2 if rows > n_rows else 0) | (4 if used < 0 or used + taken > len(free) else 0)
    pos, slot = np.zeros(n_rows, np.int64), np.full(n_rows, -1, np.int64)
    if err:
        return np.array(lens), np.zeros(R + 1, np.int64), pos, slot, np.array([0, 0, err, used]), table
    start, at, t = [0], used, 0
    for r, (l, n) in enumerate(zip(lens, new)):
        for b in range(-(-l // block), -(-(l + n) // block)):
            table[r, b] = free[at]
            at += 1
        for p in range(l, l + n):
            s = table[r, p // block]
            pos[t], slot[t] = p, s * block + p % block if 0 <= s < n_slots else -1
            t += 1
        start.append(t)
    return np.array(lens) + np.array(new), np.array(start), pos, slot, np.array([t, at - used, 0, at]), table


def attention(q, row_start, lens, table, pool, block, Hkv, at=0, scale=None):
    """(out, size, reach, most keys, values' largest) of all rows in 64 bits, as kv4_reference.attention; rows of no request: NaN."""
    n_rows, Hq, d = q.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, size, reach, most, top = np.full(q.shape, np.nan), np.zeros(q.shape), 0.0, 1, np.zeros(1)
    for r in range(len(lens)):
        lo, hi = row_start[r], row_start[r + 1]
        if hi == lo:
            continue
        n, length = hi - lo, int(lens[r])
        k, v = values(pool, table[r], length, block, Hkv, d, at) if length else np.zeros((2, 0, Hkv, d))
        there = np.array([0 <= table[r][j // block] < pool.shape[0] for j in range(length)], bool)
        p = length - n + np.arange(n)
        seen = there[None] & (np.arange(length)[None] <= p[:, None])
        o, s, x = kv4_reference.attention(q[lo:hi], k, v, seen, scale)
        out[lo:hi], size[lo:hi], reach, most = o, s, max(reach, x), max(most, length)
        used = v[:p[-1] + 1][there[:p[-1] + 1]] if length else v
        if used.size:
            top = np.maximum(top, np.nanmax(np.abs(used)))
    return out, size, reach, most, top


def attention_bound(ref, dtype):
    out, size, reach, most, top = ref
    d = out.shape[2]
    return kv4_reference.attention_bound(np.nan_to_num(out), size, reach, most, d, dtype, top)
