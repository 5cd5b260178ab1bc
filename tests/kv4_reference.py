"""A cache in 4 bits and the attention over it, plainly and in 64 bits: what the tests of these operators compare with."""
import math

import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x: np.ndarray):
    """x[.., d] float64 -> codes [.., d] (0..15) and bytes [.., d / 32] (e + 127; 255: not finite)."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    most = np.abs(g).max(-1)
    # the smallest e in range with most < 7 * 2^e (125: what is above is the largest value)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.where(most > 0, most / 7.0, 1.0))) + 1
    e = np.where(most > 0, e, -125)
    e = np.where(most >= 7.0 * np.exp2(e), e + 1, e)                 # (log2 may be off by a rounding)
    e = np.where((most > 0) & (most < 7.0 * np.exp2(e - 1)), e - 1, e)
    e = np.clip(e, -125, 125).astype(np.int64)
    y = np.abs(g) / np.exp2(e.astype(np.float64))[..., None]
    dist = np.abs(y[..., None] - GRID)
    near = dist.min(-1, keepdims=True)
    tie = dist == near                                               # (exact: y is a float times a power of two)
    code = np.where(tie & (np.arange(8) % 2 == 0), np.arange(8), -1).max(-1)
    code = np.where(code < 0, tie.argmax(-1), code)
    code = code + 8 * np.signbit(g)
    return code.reshape(x.shape), np.where(bad, 255, e + 127)


def values(code: np.ndarray, byte: np.ndarray) -> np.ndarray:
    v = np.where(code >= 8, -GRID[code % 8], GRID[code % 8]).reshape(*byte.shape, 32)
    scale = np.where(byte == 255, np.nan, np.exp2(np.where(byte == 255, 0, byte) - 127.0))
    return (v * scale[..., None]).reshape(code.shape)


def cached(x: np.ndarray) -> np.ndarray:
    """What x stands for once it is held in 4 bits."""
    return values(*quantise(x))


def slot_bytes(block, heads, d):
    return -(-block * heads * (d + d // 16) // 16) * 16


def pack(k: np.ndarray, v: np.ndarray, block: int) -> np.ndarray:
    """k, v[n, H, d] float64 -> slots [n_blocks, slot_bytes] uint8 of their blocks; rows behind the last one are zero bytes."""
    n, H, d = k.shape
    nb = -(-n // block)
    out = np.zeros((nb, slot_bytes(block, H, d)), np.uint8)
    c = H * block * (d // 2)
    s = H * block * (d // 32)
    for x, at, sat in ((k, 0, 2 * c), (v, c, 2 * c + s)):
        code, byte = quantise(x)
        for b in range(nb):
            rows = min(block, n - b * block)
            cb = np.zeros((H, block, d // 2), np.uint8)
            sb = np.zeros((H, block, d // 32), np.uint8)
            part = code[b * block:b * block + rows].transpose(1, 0, 2)
            cb[:, :rows] = part[..., 0::2] + 16 * part[..., 1::2]
            sb[:, :rows] = byte[b * block:b * block + rows].transpose(1, 0, 2)
            out[b, at:at + c] = cb.reshape(-1)
            out[b, sat:sat + s] = sb.reshape(-1)
    return out


def attention(q, k, v, seen, scale):
    """q[m, Hq, d], k, v[n, Hkv, d], seen[m, n] -> (out, magnitude of what is summed, largest sum of |q_c k_c| * scale): 64 bits.  A row that sees nothing is zero."""
    m, Hq, d = q.shape
    G = Hq // k.shape[1]
    out, size, reach = np.zeros((m, Hq, d)), np.zeros((m, Hq, d)), 0.0
    for h in range(Hq):
        kk, vv = k[:, h // G], v[:, h // G]
        for i in range(m):
            at = np.nonzero(seen[i])[0]
            if not len(at):
                continue
            s = (kk[at] @ q[i, h]) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], size[i, h] = p @ vv[at], p @ np.abs(vv[at])
            reach = max(reach, float((np.abs(kk[at]) @ np.abs(q[i, h])).max()) * scale)
    return out, size, reach


def attention_bound(out, size, reach, n, d, dtype, v=None):
    """How far an output may be off.  Scores: sums of d products in float32, off by (d + 8) half steps of the sum of magnitudes, and the scaling into the base-2 domain, the
    difference to the maximum and the exponential by four of the score's size each; a relative error r of all weights moves the result by 2 r of the summed magnitudes.
    The sum over n keys and its rescaling: n + 16 half steps.  bfloat16: each weight is rounded once (half a step, 2^-8), and so is the output.
    v: the values.  A weight below the smallest normal float32, 2^-126 of the largest weight's 1, may count as zero: n of them times the largest value."""
    half = 2.0 ** -24
    r = ((d + 8) + 12) * half * reach + 8 * half
    bound = (2 * r + (n + 16) * half) * size
    if v is not None and v.size:
        bound = bound + n * 2.0 ** -126 * np.abs(v).max()
    if dtype == torch.bfloat16:
        return bound + 2.0 ** -8 * size + 2.0 ** -8 * (np.abs(out) + bound + 2.0 ** -8 * size)
    return bound + half * np.abs(out)


def to64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().to(torch.float64).numpy()


def within(got: torch.Tensor, want: np.ndarray, bound: np.ndarray):
    """|got - want| <= bound everywhere; says where it is worst."""
    err = np.abs(to64(got) - want)
    share = np.where(err == 0, 0.0, err / np.maximum(bound, 1e-300))
    at = np.unravel_index(np.argmax(np.where(np.isnan(share), np.inf, share)), share.shape)
    print(f"   largest error / bound {share[at]:.3f}", flush=True)
    assert share[at] <= 1, f"{at}: {to64(got)[at]} instead of {want[at]}, bound {bound[at]}"
