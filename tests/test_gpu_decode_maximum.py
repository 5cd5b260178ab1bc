"""A decoded token's attention where a few keys' logits tower over the others': the softmax's maximum is that of all keys, whichever key of its group of 16 has it."""
import math

import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("place", [0, 3, 4, 9, 14, 20, 31])
@pytest.mark.parametrize("kv4", [False, True])
def test_one_key_towers_over_the_others(slim, kv4, place, dtype):
    """Logits of +-200: exponentials relative to anything but the largest overflow."""
    n, block, Hq, Hkv, d = 256, 64, 8, 2, 128
    g = np.random.default_rng(place)
    k = torch.full((n, Hkv, d), -1.0)
    k[place::32] = 1.0
    v = torch.from_numpy(g.standard_normal((n, Hkv, d)).astype(np.float32)).to(dtype)
    k = k.to(dtype)
    q = torch.full((Hq, d), 200.0 * math.sqrt(d) / d).to(dtype)
    order = torch.arange(n // block, dtype=torch.int32).cuda()
    if kv4:
        pool = torch.zeros(n // block, slim.kv4_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
        slim.slim_kv4_write(k.cuda(), v.cuda(), pool, block)
        out = slim.slim_decode_attn_kv4(q.cuda(), pool, order, block, n, Hkv)
        kk, vv = ref.cached(ref.to64(k)), ref.cached(ref.to64(v))
    else:
        pool = torch.stack([torch.stack([k[b * block:(b + 1) * block], v[b * block:(b + 1) * block]]) for b in range(n // block)]).contiguous()
        out = slim.slim_decode_attn(q.cuda(), pool.cuda(), order, block, n, Hkv)
        kk, vv = ref.to64(k), ref.to64(v)
    want, size, reach = ref.attention(ref.to64(q)[None], kk, vv, np.ones((1, n), bool), 1 / math.sqrt(d))
    ref.within(out, want[0], ref.attention_bound(want, size, reach, n, d, dtype, vv)[0])
