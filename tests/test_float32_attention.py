"""float32 attention runs in bfloat16 matrix instructions, three terms a number and six of the nine products (csrc/row_tile.h).  The bound here is near enough to what these six can do that
one product less is seen; without a GPU, both are computed and compared with it."""
import math

import numpy as np
import pytest
import torch

from tests import kv4_reference as ref
from tests.test_gpu_kv4 import F32, keys, pool_of, rand
from tests.test_gpu_sliding import inputs_of, visible

U = 2.0 ** -24                                            # half a step of a float32


def answer(q, k, v, seen, scale):
    """q[m, Hq, d], k, v[n, Hkv, d] float64 -> (result, bound).  With the products x_c = scale * q_c k_jc of key j, A_j the sum of their magnitudes, B_j the root of the sum of their squares,
    s_j their sum, the logit, and m the largest logit: s_j is off by r_j <= 8.1 U A_j + 3 sqrt(d) U (|s_j| + 2 B_j) + 12 U (m - s_j) + 8 U.
      8.1: the products left out.  A number's terms hold its first 8, next 8 and last 8 bits, cut: the second is below 2^-7 of it, the third below 2^-15, so the three products of a second
           or third term with a third lie below 2^-22, 2^-22 and 2^-30 of the numbers' product: 2^-21 = 8 U and a little;
      3 sqrt(d): d roundings, half a step of a running sum each, signs independent: five standard deviations of U / sqrt(3).  The running sum of numbers whose signs are independent is about
           B_j from its straight way to s_j;
      12: the scale, the difference to the largest logit and the exponential's argument, which all see the difference (what is common to a row cancels); 8: the exponential.
    The result's weights p_j (1 +- r_j) / sum: off by sum_j p_j r_j (|v_j| + |result|); the sum of n weighted values by 8.1 U, 3 sqrt(n) U and 16 U of its magnitudes, and U for the result."""
    m_rows, Hq, d = q.shape
    G, n = Hq // k.shape[1], k.shape[0]
    out, bound = np.zeros((m_rows, Hq, d)), np.zeros((m_rows, Hq, d))
    for h in range(Hq):
        kk, vv = k[:, h // G], v[:, h // G]
        s = np.where(seen, (q[:, h] @ kk.T) * scale, -np.inf)
        m = s.max(1, keepdims=True)
        p = np.exp(s - m)
        p /= p.sum(1, keepdims=True)
        size, spread = scale * (np.abs(q[:, h]) @ np.abs(kk).T), scale * np.sqrt(q[:, h] ** 2 @ (kk ** 2).T)
        r = np.where(seen, 8.1 * U * size + 3 * math.sqrt(d) * U * (np.abs(s) + 2 * spread) + 12 * U * (m - s) + 8 * U, 0)
        out[:, h] = p @ vv
        bound[:, h] = (p * r) @ np.abs(vv) + (p * r).sum(1, keepdims=True) * np.abs(out[:, h]) + (24.1 + 3 * math.sqrt(n)) * U * (p @ np.abs(vv)) + U * np.abs(out[:, h])
    return out, bound + n * 2.0 ** -126 * np.abs(v).max()


def terms(x):
    """The three bfloat16 numbers that add up to a float32, in float64."""
    out, r = [], x.astype(np.float32)
    for _ in range(3):
        t = (r.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
        out.append(t.astype(np.float64))
        r = r - t
    return out


def in_terms(q, k, v, seen, scale, most):
    """The attention with the products of terms a and b with a + b <= most, everything else in 64 bits."""
    def product(x, y):
        return sum(a @ b for i, a in enumerate(terms(x)) for j, b in enumerate(terms(y)) if i + j <= most)
    G, out = q.shape[1] // k.shape[1], np.zeros(q.shape)
    for h in range(q.shape[1]):
        s = np.where(seen, product(q[:, h], np.ascontiguousarray(k[:, h // G].T)) * scale, -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        out[:, h] = product(p, v[:, h // G]) / p.sum(1, keepdims=True)
    return out


CASES = [
    # n_q, n_k, Hq, Hkv, d, window, first tokens
    (1, 700, 28, 4, 128, 700, 0),
    (1, 5000, 4, 2, 64, 3000, 33),                        # the keys dealt to several workgroups
    (100, 100, 4, 2, 64, 33, 3),
    (100, 100, 3, 3, 32, 1000, 0),
    (520, 520, 4, 1, 128, 520, 0),
    (300, 700, 32, 8, 128, 260, 7),
    (9, 3001, 28, 4, 128, 3001, 0),
]


def case(n_q, n_k, Hq, Hkv, d, window, sinks):
    q, k, v = inputs_of(n_q, n_k, Hq, Hkv, d, F32, n_q + n_k)
    return q, k, v, visible(n_q, n_k, window, sinks)


@pytest.mark.parametrize("shape", CASES)
def test_the_bound_tells_six_products_from_three(shape):
    q, k, v, seen = case(*shape)
    args = [ref.to64(x) for x in (q, k, v)] + [seen, 1 / math.sqrt(shape[4])]
    want, bound = answer(*args)
    six, three = (float((np.abs(in_terms(*args, most) - want) / bound).max()) for most in (2, 1))
    print(f"six products {six:.3f} of the bound, three {three:.2f}")
    assert six < 0.25 and three > 1


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


@pytest.mark.gpu
@pytest.mark.parametrize("shape", CASES)
def test_sliding(slim, shape):
    q, k, v, seen = case(*shape)
    want, bound = answer(*(ref.to64(x) for x in (q, k, v)), seen, 1 / math.sqrt(shape[4]))
    ref.within(slim.slim_sliding_attn(q.cuda(), k.cuda(), v.cuda(), shape[5], shape[6]), want, bound)


DECODE = [(1000, 64, 28, 4, 33), (64, 64, 4, 1, 0), (5000, 16, 32, 8, 301), (40, 80, 16, 1, 900)]      # prompt tokens, block, heads, response tokens


def decode_case(n, block, Hq, Hkv, resp):
    k, v = keys(n, Hkv, 128, F32, n), rand((n, Hkv, 128), F32, n + 1)
    kr, vr = keys(resp, Hkv, 128, F32, n + 2), rand((resp, Hkv, 128), F32, n + 3)
    q = rand((Hq, 128), F32, n + 4, 0.6)
    kk, vv = (np.concatenate([ref.cached(ref.to64(a)), ref.to64(b)]) for a, b in ((k, kr), (v, vr)))
    return (k, v, kr, vr, q), (ref.to64(q)[None], kk, vv, np.ones((1, n + resp), bool), 1 / math.sqrt(128))


@pytest.mark.parametrize("shape", DECODE)
def test_the_bound_tells_three_terms_from_two_over_a_cache_in_4_bits(shape):
    """What comes from 4 bits is one term; the Query's and the weights' third ones count."""
    _, args = decode_case(*shape)
    want, bound = answer(*args)
    whole, two = (float((np.abs(in_terms(*args, most) - want) / bound).max()) for most in (2, 1))
    print(f"three terms {whole:.3f} of the bound, two {two:.2f}")
    assert whole < 0.25 and two > 1


@pytest.mark.gpu
@pytest.mark.parametrize("shape", DECODE)
def test_decode(slim, shape):
    n, block, Hq, Hkv, resp = shape
    (k, v, kr, vr, q), args = decode_case(*shape)
    want, bound = answer(*args)
    order = np.random.default_rng(n).permutation(-(-n // block)).astype(np.int32)
    pool = pool_of(slim, k, v, block, len(order), order, 1)
    out = slim.slim_decode_attn_kv4(q.cuda(), pool, torch.from_numpy(order).cuda(), block, n, Hkv, kr.cuda() if resp else None, vr.cuda() if resp else None)
    ref.within(out, want[0], bound[0])
