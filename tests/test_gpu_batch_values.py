"""Attention of a batch over blocks whose Values differ widely, on the GPU, against 64 bits: what a key's block holds beside it, and what a row does not see, must not cost the row its result."""
import math

import numpy as np
import pytest
import torch

from tests import batch_reference as ref
from tests.kv4_reference import to64, within
from tests.test_gpu_kv4 import rand

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def attend(slim, q, k, v, block, rows_see=None):
    """(result, 64-bit reference) of the last len(q) of the tokens k, v."""
    n, Hkv, d = k.shape
    nb = -(-n // block)
    pool = torch.zeros(nb, slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(np.arange(n)))
    out = slim.slim_batch_attn_kv8(q.cuda(), i32([0, len(q)]), i32([n]), i32([np.arange(nb)]), pool, block, Hkv)
    return out, ref.attention(to64(q), [0, len(q)], [n], np.arange(nb)[None], pool.cpu().numpy(), block, Hkv)


# Rows of a kv head: 4 a query; above 64 they go in tiles of 256.
MANY = [(40, 64, BF16), (40, 128, BF16), (140, 128, BF16), (9, 128, BF16), (40, 64, F32)]


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("power", [6, 12, 13, 16, 20, 23, 26, 29, 60, 110])
def test_a_token_of_little_weight_and_large_values(slim, n, d, dtype, power):
    """Flat scores and Values about 1, one token with Values of 2^power whose weight is 10^-15 (2^-80 for the largest): it adds little, and its block's exponent must not push the others out."""
    tokens, block, Hq, Hkv = 640, 64, 8, 2
    v = rand((tokens, Hkv, d), F32, power) * 0.2 + 1.0
    v[5] = 2.0 ** power
    k = torch.zeros(tokens, Hkv, d)
    k[5, :, 0] = -1.0
    q = torch.zeros(n, Hq, d)
    q[:, :, 0] = (math.log(1e15) if power < 40 else 140 * math.log(2)) * math.sqrt(d)
    q = q.to(dtype)
    out, want = attend(slim, q, k, v, block)
    within(out, want[0], ref.attention_bound(want, dtype))


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("power", [13, 29, 100])
def test_a_later_token_with_large_values(slim, n, d, dtype, power):
    """A token that only the last rows see raises its block's exponent: the rows in front of it do not see it, and have the mean of the others."""
    held, block, Hq, Hkv = 700, 64, 8, 2
    tokens = held + n
    v = rand((tokens, Hkv, d), F32, 1) * 0.2 + 1.0
    later = tokens - 3
    v[later] = 2.0 ** power
    k = rand((tokens, Hkv, d), F32, 2) * 0.1
    q = rand((n, Hq, d), F32, 3).to(dtype)
    out, want = attend(slim, q, k, v, block)
    within(out, want[0], ref.attention_bound(want, dtype))
    assert (out[:n - 3].float() < 1.5).all()


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("tokens", [512, 9000])
@pytest.mark.parametrize("sizes", [[0.0, 1e20], [0.0, 1.0, 1e20, 1e30], [1e-30, 1e30], [0.0, 1.0]])
def test_blocks_of_zeros_count_in_the_sum(slim, n, d, dtype, tokens, sizes):
    """Equal scores, blocks with Values of 0 to 10^30 in turn: each key counts once, whatever its block's exponent."""
    block, Hq, Hkv = 16, 8, 2
    v = (rand((tokens, Hkv, d), F32, 2) * 0.2 + 1.0) * torch.tensor(sizes)[torch.arange(tokens) // block % len(sizes)][:, None, None]
    q = rand((n, Hq, d), F32, 3).to(dtype)
    out, want = attend(slim, q, torch.zeros(tokens, Hkv, d), v, block)
    within(out, want[0], ref.attention_bound(want, dtype))


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("tokens", [900, 9000])
def test_rows_that_look_at_one_kind_of_block(slim, n, d, dtype, tokens):
    """Blocks with Values of 10^-30 to 10^30, and queries that look at one kind each, some 86 binary places above the others: results of every size beside each other."""
    block, Hq, Hkv = 16, 8, 2
    sizes = [1.0, 1e-30, 1e20, 1e-12, 1e30, 1e6]
    kind = np.arange(tokens) // block % len(sizes)
    v = rand((tokens, Hkv, d), F32, 2) * torch.tensor(sizes)[kind][:, None, None]
    k = rand((tokens, Hkv, d), F32, 3) * 0.1
    k[torch.arange(tokens), :, kind] += 8.0
    q = rand((n, Hq, d), F32, 4) * 0.1
    q[:, :, :len(sizes)] = 0.0
    for i in range(n):
        for h in range(Hq):
            q[i, h, (i + h) % len(sizes)] = 60.0 * math.sqrt(d / 64)
    q = q.to(dtype)
    out, want = attend(slim, q, k, v, block)
    bound = ref.attention_bound(want, dtype)
    rest = want[3] * 2.0 ** -126 * want[4].max()         # what weights below the smallest normal number leave out is of the largest Values' size
    assert rest < 1e-3
    within(out, want[0], bound)
