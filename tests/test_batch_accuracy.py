"""How exact the attention over blocks in 8 bits is (csrc/kv8.hip): bounds that follow from how its weights are rounded, near enough that weights with fewer places are seen.  Without a GPU, the
roundings are formed and compared with the bounds; on it, the operator."""
import math

import numpy as np
import pytest
import torch

from tests import batch_reference as ref
from tests.kv4_reference import to64, within
from tests.test_float32_attention import U, answer, in_terms
from tests.test_gpu_kv4 import keys, rand

BF16, F32 = torch.bfloat16, torch.float32
HALF, TWO = 2.0 ** -11, 2.0 ** -17                        # of a weight: half a step of a float16; of what a bfloat16 leaves, in a second one


def bf16(x):
    """x float64 -> the nearest bfloat16 numbers."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def bound_of(args, weight):
    """q, k, v, seen, scale in 64 bits -> (result, bound) of bfloat16 outputs: what float32 arithmetic leaves (answer), `weight` of the weighted magnitudes, for float16 2^-34 of the magnitudes (a
    weight below the normal ones is off by half a step, 2^-25, where the row's largest is 2^9 at least), and the output's rounding, half a step of the numbers around it."""
    q, k, v, seen, scale = args
    want, bound = answer(*args)
    G = q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        s = np.where(seen, (q[:, h] @ k[:, h // G].T) * scale, -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        bound[:, h] += weight * (p @ np.abs(v[:, h // G])) / p.sum(1, keepdims=True) + (2.0 ** -34 * (seen @ np.abs(v[:, h // G])) if weight == HALF else 0)
    return want, bound + np.ldexp(1.0, np.frexp(np.abs(want) + bound)[1] - 9)


def rounded(args, how):
    """The attention with weights rounded by `how` (of the largest, 1), the sum not, the output once; everything else in 64 bits."""
    q, k, v, seen, scale = args
    out = np.zeros(q.shape)
    for h in range(q.shape[1]):
        g = h // (q.shape[1] // k.shape[1])
        s = np.where(seen, (q[:, h] @ k[:, g].T) * scale, -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        out[:, h] = bf16(how(p) @ v[:, g] / p.sum(1, keepdims=True))
    return out


def half(p):
    return (p * 2.0 ** 10).astype(np.float16).astype(np.float64) * 2.0 ** -10


def two(p):
    return bf16(p) + bf16(p - bf16(p))


CASES = [
    # tokens held, rows, block, Hq, Hkv, d, powers of the blocks' Values, weights
    (700, 1, 64, 28, 4, 128, 0, TWO),                     # tiles of 16 rows
    (3000, 2, 16, 8, 2, 64, 0, TWO),
    (300, 6, 64, 8, 2, 128, 0, TWO),                      # of 32
    (900, 13, 48, 8, 2, 64, 20, TWO),
    (500, 60, 64, 8, 2, 128, 0, HALF),                    # of 256
    (300, 90, 16, 8, 2, 64, 0, HALF),
    (2000, 40, 64, 28, 4, 128, 8, HALF),
    # Of 256, exponents of all blocks too far apart for one float16: a workgroup looks at those of its own stretch of the keys, from 256 of them on, four or eight blocks here, and they may lie
    # within 12 of each other, so that the weights are float16 there
    (2000, 40, 64, 8, 2, 128, 14, HALF),
    (700, 60, 32, 8, 2, 64, 20, HALF),
    # every other block's Values are 2^-16, 2^-20, 2^-14 times its neighbours', and every stretch has two blocks at least
    (1200, 40, 64, 8, 2, 128, -16, TWO),
    (700, 60, 32, 8, 2, 64, -20, TWO),
    (1100, 170, 32, 8, 2, 128, -14, TWO),
]


def make(held, rows, block, Hq, Hkv, d, powers, dtype, spread=1.5):
    """(q, pool, 64-bit arguments): Values of the blocks up to 2^powers apart (below zero: every other block), scores of `spread` deviations, so that few keys make most of a row."""
    n = held + rows
    nb = -(-n // block)
    g = np.random.default_rng(n + d)
    v = rand((n, Hkv, d), F32, n + 1).double().numpy() * np.exp2(np.round(g.random(nb) * powers) if powers >= 0 else np.arange(nb) % 2 * powers)[np.arange(n) // block][:, None, None]
    k = keys(n, Hkv, d, F32, n).double().numpy()
    q = rand((rows, Hq, d), dtype, n + 2)
    q = (q * (spread * math.sqrt(d) / float((q.double().reshape(-1, d) @ torch.from_numpy(k[:, 0]).T).std()))).to(dtype)
    pool = ref.write(np.zeros((nb, ref.slot_bytes(block, Hkv, d)), np.uint8), k, v, np.arange(n), block)
    kk, vv = ref.values(pool, np.arange(nb), n, block, Hkv, d)
    return q, pool, (to64(q), kk, vv, np.arange(n)[None] <= held + np.arange(rows)[:, None], 1 / math.sqrt(d))


@pytest.mark.parametrize("case", CASES)
def test_the_bound_tells_the_weights_places(case):
    _, pool, args = make(*case[:7], BF16)
    if case[1] * case[3] // case[4] > 64 and case[7] == TWO:
        e = np.stack([ref.parts(x, case[2], case[4], case[5])[2][:, 1] for x in pool]).astype(int)
        assert (np.abs(np.diff(e, axis=0)) > 12).all()
    want, bound = bound_of(args, case[7])
    share = {name: float((np.abs(rounded(args, how) - want) / bound).max()) for name, how in (("one", bf16), ("two", two), ("half", half))}
    print(share)
    assert share["one"] > 1.2 and share["two"] < 1.0
    assert share["half"] < 1.0 if case[7] == HALF else share["half"] > 1.0


def answer32(args):
    """(result, bound) of float32 rows as `answer`, without what it allows for products that are left out: Keys and Values from 8 bits are one term, whose products with all three of a Query's or
    a weight's, cut, are kept."""
    q, k, v, seen, scale = args
    want, bound = answer(*args)
    for h in range(q.shape[1]):
        kk, vv = k[:, h // (q.shape[1] // k.shape[1])], v[:, h // (q.shape[1] // k.shape[1])]
        s = np.where(seen, (q[:, h] @ kk.T) * scale, -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        r = np.where(seen, 8.1 * U * scale * (np.abs(q[:, h]) @ np.abs(kk).T), 0)
        bound[:, h] -= (p * r) @ np.abs(vv) + (p * r).sum(1, keepdims=True) * np.abs(want[:, h]) + 8.1 * U * (p @ np.abs(vv))
    return want, bound


F32_CASES = [(700, 40, 64, 28, 4, 128), (1500, 60, 16, 8, 2, 64), (300, 90, 64, 8, 2, 128)]      # (with scores of 6 deviations: the Query's third term counts most)


@pytest.mark.parametrize("case", F32_CASES)
def test_the_bound_tells_three_terms_from_two(case):
    """What comes from 8 bits is one term; the Query's and the weights' third ones count."""
    _, _, args = make(*case, 0, F32, 6.0)
    want, bound = answer32(args)
    whole, fewer = (float((np.abs(in_terms(*args, most) - want) / bound).max()) for most in (2, 1))
    print(f"three terms {whole:.3f} of the bound, two {fewer:.2f}")
    assert whole < 0.25 and fewer > 1


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def attend(slim, case, q, pool):
    held, rows, block, Hkv = case[0], case[1], case[2], case[4]
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()
    return slim.slim_batch_attn_kv8(q.cuda(), i32([0, rows]), i32([held + rows]), i32(np.arange(len(pool)))[None], torch.from_numpy(pool).cuda(), block, Hkv)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES)
def test_bfloat16(slim, case):
    q, pool, args = make(*case[:7], BF16)
    within(attend(slim, case, q, pool), *bound_of(args, case[7]))


@pytest.mark.gpu
@pytest.mark.parametrize("case", F32_CASES)
def test_float32(slim, case):
    q, pool, args = make(*case, 0, F32, 6.0)
    within(attend(slim, case, q, pool), *answer32(args))
