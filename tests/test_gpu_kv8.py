"""Rows of a batch written into a pool of blocks in 8 bits and read back, on the GPU, against a plain implementation in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import batch_reference as ref
from tests.kv4_reference import to64
from tests.test_gpu_kv4 import keys, rand, same

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def equal_pools(got, want):
    got = got.cpu().numpy()
    bad = np.argwhere(got != want)
    assert not len(bad), (len(bad), [(tuple(b), got[tuple(b)], want[tuple(b)]) for b in bad[:8]])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_rounding(slim, dtype):
    """Blocks of every size of largest magnitude, filled with the values, the borders between them and their neighbours."""
    eps = torch.finfo(dtype).eps
    marks = np.concatenate([ref.GRID, (ref.GRID[1:] + ref.GRID[:-1]) / 2, [447.0, 449.0, 1e-3, 1e-5]])
    marks = np.concatenate([marks, marks * (1 + eps), marks * (1 - eps / 2)])
    marks = marks[marks <= 448][:768]
    blocks = []
    for e in list(range(-140, 120, 3)) + [-118, -117, -116, 117, 118, 119, 120]:
        for top in (448.0, 256.0, 300.0, 224.0 * (1 + eps)):
            m = np.resize(marks, 16 * 64) * np.where(np.arange(16 * 64) % 3 == 1, -1, 1)
            x = np.clip(m, -top, top) * 2.0 ** e
            x[7] = -top * 2.0 ** e
            blocks.append(x.reshape(16, 1, 64))
    with np.errstate(over="ignore"):
        x = torch.from_numpy(np.concatenate(blocks)).to(F32).to(dtype)
    x = torch.where(torch.isfinite(x), x, torch.full_like(x, torch.finfo(dtype).max))
    n = x.shape[0]
    pool = torch.zeros(n // 16, slim.kv8_block_bytes(16, 1, 64), dtype=torch.uint8, device="cuda")
    y = x.flip(0).contiguous()
    assert slim.slim_kv8_write(x.cuda(), y.cuda(), pool, 16, i32(np.arange(n))) is pool
    want = ref.write(np.zeros(pool.shape, np.uint8), to64(x), to64(y), np.arange(n), 16)
    equal_pools(pool, want)
    k, v = slim.slim_kv8_read(pool, 16, n, n_kv_heads=1, head_dim=64, dtype=dtype)
    kk, vv = ref.values(want, np.arange(n // 16), n, 16, 1, 64)
    same(k, kk)
    same(v, vv)


def batch(lens, new, block, n_slots, seed):
    """(places of the step's rows, tables) of requests whose blocks lie in slots in no order."""
    g = np.random.default_rng(seed)
    order, at, places, tables = g.permutation(n_slots), 0, [], []
    for l, n in zip(lens, new):
        nb = -(-(l + n) // block)
        mine = order[at:at + nb]
        at += nb
        tables.append(mine)
        p = np.arange(l, l + n)
        places.append(mine[p // block] * block + p % block)
    return np.concatenate(places), tables


@pytest.mark.parametrize("lens,new,block,H,d,dtype", [
    ([0], [1], 16, 1, 64, BF16), ([0], [1], 16, 8, 128, F32), ([15], [1], 16, 2, 128, BF16), ([63], [2], 64, 8, 128, BF16), ([0], [200], 64, 8, 128, BF16),
    ([5, 0, 31, 16, 100], [1, 1, 1, 1, 1], 32, 4, 128, BF16), ([7, 0, 0, 300], [150, 3, 65, 33], 80, 4, 128, F32), ([3, 4], [130, 40], 1, 2, 64, BF16),
    ([11, 2], [129, 5], 7, 3, 64, F32), ([0, 100], [1000, 333], 300, 2, 128, BF16), ([250], [65], 300, 2, 64, BF16), ([0], [700], 1000, 2, 128, F32),
    (list(range(40)), [1] * 40, 16, 8, 128, BF16), ([9] * 300, [1 + i % 3 for i in range(300)], 16, 2, 64, BF16), ([0] * 30, [37] * 30, 16, 8, 128, BF16),
    ([0] * 3, [9000, 40, 7000], 64, 2, 128, BF16)])
def test_write_and_read_back(slim, lens, new, block, H, d, dtype):
    print(f"kv8 write lens={lens[:5]} new={new[:5]} block={block} H={H} d={d} {dtype}", flush=True)
    n = sum(new)
    g = np.random.default_rng(n + block)
    n_slots = sum(-(-(l + m) // block) for l, m in zip(lens, new)) + 3
    places, tables = batch(lens, new, block, n_slots, n)
    size, at = ref.slot_bytes(block, H, d), 48
    before = g.integers(0, 256, (n_slots, at + size + 32)).astype(np.uint8)
    # what the blocks hold already: exponents around those of the rows that come
    view = before[:, at + 2 * H * block * d:at + 2 * H * block * d + 2 * H]
    view[:] = g.integers(114, 130, view.shape)
    k, v = keys(n, H, d, dtype, n), keys(n, H, d, dtype, n + 1)
    qkv = torch.full((n, 2 * H + 3, d), 7.0, dtype=dtype)
    qkv[:, 1:H + 1], qkv[:, H + 2:2 * H + 2] = k, v
    qkv = qkv.cuda()
    pool = torch.from_numpy(before).cuda()
    slim.slim_kv8_write(qkv[:, 1:H + 1], qkv[:, H + 2:2 * H + 2], pool, block, i32(places), layer_offset=at)
    want = ref.write(before, to64(k), to64(v), places, block, at)
    equal_pools(pool, want)
    # each request's rows, into rows that are apart
    for r in (0, len(lens) - 1):
        m = lens[r] + new[r]
        wide = torch.full((m + 2, H + 2, d), 7.0, dtype=dtype, device="cuda")
        kr, vr = slim.slim_kv8_read(pool, block, m, i32(tables[r]), k_out=wide[:m, :H], v_out=torch.empty(m, H, d, dtype=dtype, device="cuda"), layer_offset=at)
        kk, vv = ref.values(want, tables[r], m, block, H, d, at)
        same(kr, kk)
        same(vr, vv)
        assert (wide[m:] == 7).all() and (wide[:, H:] == 7).all()


def test_token_by_token_the_exponent_only_grows(slim):
    """A block filled by 40 writes; every state of the pool."""
    block, H, d = 32, 2, 64
    g = np.random.default_rng(0)
    x = g.standard_normal((40, H, d)) * np.exp2(g.integers(-12, 4, (40, H, 1)))
    x[5, 0], x[20, 1] = 0.0, 1e30
    k, v = torch.from_numpy(x).to(BF16), torch.from_numpy(x[::-1].copy()).to(BF16)
    pool = torch.zeros(2, slim.kv8_block_bytes(block, H, d), dtype=torch.uint8, device="cuda")
    want = pool.cpu().numpy()
    for t in range(40):
        slim.slim_kv8_write(k[t:t + 1].cuda(), v[t:t + 1].cuda(), pool, block, i32([t]))
        want = ref.write(want, to64(k[t:t + 1]), to64(v[t:t + 1]), [t], block)
        equal_pools(pool, want)
    # and a block that begins anew forgets what it held
    slim.slim_kv8_write(k[:3].cuda() * 1e-3, v[:3].cuda() * 1e-3, pool, block, i32([0, 1, 2]))
    equal_pools(pool, ref.write(want, to64(k[:3] * 1e-3), to64(v[:3] * 1e-3), [0, 1, 2], block))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_numbers_that_are_not_finite(slim, dtype):
    """They read back as NaN, alone, and do not count for the exponent; also where they were there before, and were rounded again."""
    block, H, d = 16, 2, 64
    k = keys(40, H, d, dtype, 4)
    k[3, 0, 5], k[7, 1, 40], k[18, 0, 63], k[33, 1, 0] = math.inf, -math.inf, math.nan, torch.finfo(dtype).max
    k[20], k[36:, 1] = 0.0, math.nan
    pool = torch.zeros(3, slim.kv8_block_bytes(block, H, d), dtype=torch.uint8, device="cuda")
    want = pool.cpu().numpy()
    for a, b in ((0, 20), (20, 21), (21, 32), (32, 35), (35, 40)):
        x = k[a:b] * (64 if a == 21 else 1)
        slim.slim_kv8_write(x.cuda(), x.cuda(), pool, block, i32(np.arange(a, b)))
        want = ref.write(want, to64(x), to64(x), np.arange(a, b), block)
    equal_pools(pool, want)
    kr, vr = slim.slim_kv8_read(pool, block, 40, n_kv_heads=H, head_dim=d, dtype=dtype)
    kk, _ = ref.values(want, np.arange(3), 40, block, H, d)
    assert np.isnan(kk).sum() == 3 + 4 * d and np.array_equal(np.isnan(kk), ~np.isfinite(to64(k)))
    same(kr, kk)
    same(vr, kk)


def test_rows_and_blocks_without_a_place_are_left_out(slim):
    n, H, d, block = 100, 2, 64, 16
    k, v = keys(n, H, d, BF16, 1), keys(n, H, d, BF16, 2)
    slots = np.array([2, -1, 0, 99, 1, -7, 3])
    p = np.arange(n)
    places = np.where((slots[p // block] >= 0), slots[p // block] * block + p % block, -1)
    places[3 * block:4 * block] = np.array([2**31 - 1, 4 * block, -2**31, -16] * 4)     # outside the pool of four slots
    pool = torch.full((4, slim.kv8_block_bytes(block, H, d)), 0x5a, dtype=torch.uint8, device="cuda")
    before = pool.cpu().numpy()
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(places))
    want = ref.write(before, to64(k), to64(v), places, block)
    equal_pools(pool, want)
    ks, vs = (torch.full((n + 1, H, d), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    slim.slim_kv8_read(pool, block, n, i32(slots), k_out=ks, v_out=vs)
    kk, vv = ref.values(want, slots, n, block, H, d)
    same(ks[:n], np.where(np.isnan(kk), 7.0, kk))
    same(vs[:n], np.where(np.isnan(vv), 7.0, vv))
    assert (ks[n:] == 7).all()
    fresh, _ = slim.slim_kv8_read(pool, block, n, i32(slots), n_kv_heads=H, head_dim=d)
    same(fresh, np.nan_to_num(kk))
    # no row has a place
    now = pool.clone()
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(np.full(n, -1)))
    assert torch.equal(pool, now)


def test_pinned_host_pool(slim):
    n, H, d, block = 100, 2, 128, 16
    k, v = keys(n, H, d, BF16, 5), keys(n, H, d, BF16, 6)
    host = torch.zeros(7, slim.kv8_block_bytes(block, H, d), dtype=torch.uint8).pin_memory()
    slim.slim_kv8_write(k.cuda(), v.cuda(), host, block, i32(np.arange(n)))
    torch.cuda.synchronize()
    want = ref.write(np.zeros(host.shape, np.uint8), to64(k), to64(v), np.arange(n), block)
    equal_pools(host, want)
    kr, vr = slim.slim_kv8_read(host, block, n, n_kv_heads=H, head_dim=d)
    kk, vv = ref.values(want, np.arange(7), n, block, H, d)
    same(kr, kk)
    same(vr, vv)


def test_far_slots(slim):
    """Slots behind 4 GB, and rows 128 MB apart."""
    n, block, H, d, ld = 40, 16, 8, 128, 1 << 26
    size = slim.kv8_block_bytes(block, H, d)
    n_slots = 2**32 // size + 1000
    pool = torch.zeros(n_slots, size, dtype=torch.uint8, device="cuda")
    slots = np.array([n_slots - 1, 3, n_slots - 900])
    p = np.arange(n)
    k, v = keys(n, H, d, BF16, 1), keys(n, H, d, BF16, 2)
    room = torch.empty((n - 1) * ld + 2 * H * d, dtype=BF16, device="cuda")
    kf, vf = (room.as_strided((n, H, d), (ld, d, 1), at) for at in (0, H * d))
    kf.copy_(k)
    vf.copy_(v)
    slim.slim_kv8_write(kf, vf, pool, block, i32(slots[p // block] * block + p % block))
    want = ref.write(np.zeros((3, size), np.uint8), to64(k), to64(v), p, block)
    equal_pools(pool[torch.from_numpy(slots).cuda()], want)
    kf.zero_()
    vf.zero_()
    slim.slim_kv8_read(pool, block, n, i32(slots), k_out=kf, v_out=vf)
    kk, vv = ref.values(want, np.arange(3), n, block, H, d)
    same(kf, kk)
    same(vf, vv)


def test_binding_refusals(slim):
    k = torch.zeros(16, 2, 64, dtype=BF16, device="cuda")
    pool = torch.zeros(1, slim.kv8_block_bytes(16, 2, 64), dtype=torch.uint8, device="cuda")
    places = i32(np.arange(16))
    for bad in (lambda: slim.slim_kv8_write(k, k[:4], pool, 16, places), lambda: slim.slim_kv8_write(k, k.float(), pool, 16, places), lambda: slim.slim_kv8_write(k, k.cpu(), pool, 16, places),
                lambda: slim.slim_kv8_write(k.transpose(0, 1), k.transpose(0, 1), pool, 16, places), lambda: slim.slim_kv8_write(k, k, pool, 16, places[:8]),
                lambda: slim.slim_kv8_write(k, k, pool, 16, places.cpu()), lambda: slim.slim_kv8_write(k, k, pool.cpu(), 16, places),
                lambda: slim.slim_kv8_read(pool, 16, 16, k_out=k[:8], v_out=k[:8]), lambda: slim.slim_kv8_read(pool, 16, 16, k_out=k),
                lambda: slim.slim_kv8_read(pool, 16, 17, i32([0]), n_kv_heads=2, head_dim=64)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: slim.slim_kv8_write(k, k, pool, 16, places.long()), lambda: slim.slim_kv8_write(k.half(), k.half(), pool, 16, places),
                lambda: slim.slim_kv8_read(pool, 16, 16, torch.zeros(1, dtype=torch.int64, device="cuda"), n_kv_heads=2, head_dim=64)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: slim.slim_kv8_write(k, k, pool, 17, places), lambda: slim.slim_kv8_write(k, k, pool[:0], 16, places), lambda: slim.slim_kv8_write(k[:0], k[:0], pool, 16, places[:0]),
                lambda: slim.slim_kv8_read(pool, 16, 0, k_out=k, v_out=k), lambda: slim.slim_kv8_read(pool, 16, 16, k_out=k[:1].expand(16, 2, 64), v_out=k)):
        with pytest.raises(slim.SlimError):
            bad()
