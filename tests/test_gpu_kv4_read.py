"""Blocks in 4 bits read back into tensors that the call allocates: how many rows, and what those hold that no slot has."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref
from tests.test_gpu_kv4 import BF16, F32, keys, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def written(slim, n, H, d, block, dtype, sob=None, slots=None):
    k, v = keys(n, H, d, dtype, n), keys(n, H, d, dtype, n + 1)
    nb = -(-n // block)
    pool = torch.zeros(slots or nb, slim.kv4_block_bytes(block, H, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv4_write(k.cuda(), v.cuda(), pool, block, sob)
    return pool, ref.cached(ref.to64(k)), ref.cached(ref.to64(v))


@pytest.mark.parametrize("n,block,lists", [(74, 64, ([0], [1], [0, 1])), (65, 64, ([0], [1])), (128, 64, ([0], [1])), (205, 32, ([0, 2, 5], [0, 2, 6], [6], [5], [0, 1, 2, 3, 4, 5]))])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_row_of_the_listed_blocks(slim, n, block, lists, dtype):
    pool, k, v = written(slim, n, 2, 64, block, dtype)
    for some in lists:
        rows = np.concatenate([np.arange(b * block, min(n, (b + 1) * block)) for b in some])
        for n_out in (None, len(rows), max(1, len(rows) - 3)):
            kr, vr = slim.slim_kv4_read(pool, block, n, blocks=torch.tensor(some, dtype=torch.int32, device="cuda"), n_kv_heads=2, head_dim=64, dtype=dtype, n_out=n_out)
            same(kr, k[rows[:n_out]])
            same(vr, v[rows[:n_out]])


def test_captured_with_the_rows_given(slim):
    """Counting the rows waits for the GPU: a call in a graph says how many, or gives the outputs."""
    n, block = 205, 32
    pool, k, v = written(slim, n, 2, 64, block, BF16)
    some = torch.tensor([1, 4], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError, match="n_out"):
            slim.slim_kv4_read(pool, block, n, blocks=some, n_kv_heads=2, head_dim=64)
        kr, vr = slim.slim_kv4_read(pool, block, n, blocks=some, n_kv_heads=2, head_dim=64, n_out=64)
    for lo, hi in ((1, 4), (0, 5)):
        some.copy_(torch.tensor([lo, hi]))
        graph.replay()
        torch.cuda.synchronize()
        rows = np.concatenate([np.arange(b * block, (b + 1) * block) for b in (lo, hi)])
        same(kr, k[rows])
        same(vr, v[rows])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_no_slot_has_are_zero(slim, dtype):
    """Blocks without a slot, blocks that the prompt does not have, and rows behind the listed blocks: in outputs that the call allocates."""
    n, H, d, block = 200, 2, 128, 16
    sob = torch.arange(13, dtype=torch.int32).roll(5)
    sob[[1, 4, 12]] = torch.tensor([-1, 99, -5], dtype=torch.int32)
    pool, k, v = written(slim, n, H, d, block, dtype, sob.cuda(), 13)
    for x in (k, v):
        for b in (1, 4, 12):
            x[b * block:(b + 1) * block] = 0
    some = torch.tensor([0, 1, 3, 7, 40], dtype=torch.int32)
    lists = ((None, None, np.arange(n)), (some, 5 * block, np.r_[0:32, 48:64, 112:128]), (some[:3], 60, np.r_[0:32, 48:64]))
    for blocks, n_out, rows in lists:
        for _ in range(3):
            old = [torch.full((n_out or n, H, d), 7.0, dtype=dtype, device="cuda") for _ in range(4)]         # what the allocator hands out next
            del old
            kr, vr = slim.slim_kv4_read(pool, block, n, sob.cuda(), blocks if blocks is None else blocks.cuda(), n_kv_heads=H, head_dim=d, dtype=dtype, n_out=n_out)
            for got, x in ((kr, k), (vr, v)):
                want = np.zeros((n_out or n, H, d))
                want[:len(rows)] = x[rows]
                same(got, want)
    # a pool that holds the first blocks only, without a map
    kr, vr = slim.slim_kv4_read(pool[:5], block, n, n_kv_heads=H, head_dim=d, dtype=dtype)
    assert kr[:5 * block].any() and not kr[5 * block:].any() and not vr[5 * block:].any()
