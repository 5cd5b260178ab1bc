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
