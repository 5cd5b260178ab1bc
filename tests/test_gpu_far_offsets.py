"""The cache in 4 bits and the sliding window where addresses pass 32 bits: far slots, rows far apart, long caches, many rows."""
import math

import numpy as np
import pytest
import torch

from tests import kv4_reference as ref
from tests.test_gpu_kv4 import keys, rand, same

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def test_far_slots(slim):
    n, block, Hq, Hkv, d = 300, 64, 16, 8, 128
    size = slim.kv4_block_bytes(block, Hkv, d)
    n_slots = 2**32 // size + 1000
    nb = slim.n_blocks(n, block)
    k, v, q = keys(n, Hkv, d, BF16, 1), rand((n, Hkv, d), BF16, 2), rand((Hq, d), BF16, 3, 0.6)
    pool = torch.zeros(n_slots, size, dtype=torch.uint8, device="cuda")
    slot_of_block = torch.tensor([n_slots - 1, 3, n_slots - 900, n_slots - 7, 0], dtype=torch.int32)
    assert slot_of_block.numel() == nb
    block_of_slot = torch.full((n_slots,), -1, dtype=torch.int32)
    block_of_slot[slot_of_block.long()] = torch.arange(nb, dtype=torch.int32)
    slim.slim_kv4_write(k.cuda(), v.cuda(), pool, block, slot_of_block.cuda())
    packed = ref.pack(ref.to64(k), ref.to64(v), block)
    for b in range(nb - 1):                               # (the last block is short: its other rows are zeros in the pool)
        np.testing.assert_array_equal(pool[int(slot_of_block[b])].cpu().numpy(), packed[b])
    kr, vr = slim.slim_kv4_read(pool, block, n, slot_of_block.cuda(), n_kv_heads=Hkv, head_dim=d)
    k64, v64 = ref.cached(ref.to64(k)), ref.cached(ref.to64(v))
    same(kr, k64)
    same(vr, v64)
    out = slim.slim_decode_attn_kv4(q.cuda(), pool, block_of_slot.cuda(), block, n, Hkv)
    seen = np.ones((1, n), bool)
    want, bound, reach = ref.attention(ref.to64(q)[None], k64, v64, seen, 1 / math.sqrt(d))
    ref.within(out[None], want, ref.attention_bound(want, bound, reach, n, d, BF16, v64))


def test_rows_far_apart(slim):
    n, block, H, d, ld = 40, 16, 2, 128, 1 << 26          # 128 MB from row to row
    k, v = keys(n, H, d, BF16, 4), rand((n, H, d), BF16, 5)
    room = torch.empty((n - 1) * ld + 2 * H * d, dtype=BF16, device="cuda")
    kf, vf = (room.as_strided((n, H, d), (ld, d, 1), at) for at in (0, H * d))
    kf.copy_(k)
    vf.copy_(v)
    pool = torch.zeros(slim.n_blocks(n, block), slim.kv4_block_bytes(block, H, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv4_write(kf, vf, pool, block)
    np.testing.assert_array_equal(pool.cpu().numpy(), ref.pack(ref.to64(k), ref.to64(v), block))
    kf.zero_()
    vf.zero_()
    slim.slim_kv4_read(pool, block, n, k_out=kf, v_out=vf)
    same(kf, ref.cached(ref.to64(k)))
    same(vf, ref.cached(ref.to64(v)))


def last_rows(slim, q, k, v, window, sinks, count):
    """The last `count` rows of a call against 64 bits, from the keys that they see."""
    out = slim.slim_sliding_attn(q, k, v, window, sinks)[-count:]
    near = window + count - 1
    ks, vs = (torch.cat((x[:sinks], x[-near:])).cpu() for x in (k, v))
    d, n = q.shape[2], ks.shape[0]
    p, j = np.arange(n - count, n)[:, None], np.arange(n)[None]
    seen = (j <= p) & ((j > p - window) | (j < sinks))
    want, size, reach = ref.attention(ref.to64(q[-count:].cpu()), ref.to64(ks), ref.to64(vs), seen, 1 / math.sqrt(d))
    ref.within(out, want, ref.attention_bound(want, size, reach, int(seen.sum(1).max()), d, q.dtype, ref.to64(vs)))


def filled(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, dtype=dtype, device="cuda", generator=g)


@pytest.mark.parametrize("n_q,Hq,dtype", [(1, 32, BF16), (40, 32, BF16), (900, 64, BF16), (3, 32, F32)])
def test_long_cache(slim, n_q, Hq, dtype):
    n_k, Hkv, d = 1_200_003, 16, 128                      # Keys of 4.9 GB, or 9.8
    k, v = filled((n_k, Hkv, d), dtype, 6), filled((n_k, Hkv, d), dtype, 7)
    last_rows(slim, filled((n_q, Hq, d), dtype, 8), k, v, 500, 5, min(n_q, 20))


@pytest.mark.parametrize("n,Hq,d,dtype", [(600_011, 32, 128, BF16), (1_100_003, 32, 32, F32)])
def test_many_rows(slim, n, Hq, d, dtype):                # outputs of 4.9 and 4.5 GB
    k, v = filled((n, 2, d), dtype, 9), filled((n, 2, d), dtype, 10)
    last_rows(slim, filled((n, Hq, d), dtype, 11), k, v, 90, 3, 20)
