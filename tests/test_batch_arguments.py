"""The calls on a batch of requests: sizes, and what is refused before anything is enqueued (no GPU)."""
import ctypes

import pytest
import torch

from tests import batch_reference as ref

I32, BF16, F32 = torch.int32, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import os

    import paper_2508_06447_amd as slim
    if not os.path.exists(slim.LIB_PATH):
        from paper_2508_06447_amd.build import build_lib
        build_lib(verbose=False)
    return slim


@pytest.fixture(scope="module")
def lib(slim):
    return slim.load_library()


def at(x):                                                # addresses that are never dereferenced on these paths
    return ctypes.c_void_p(x)


NULL, ONE, ODD = at(0), at(256), at(264)
SIZE = 2 * 64 * 8 * 128 + 16


def test_block_bytes(lib):
    assert lib.slim_kv8_block_bytes(64, 8, 128) == SIZE
    for block, heads, d in ((1, 1, 64), (7, 3, 64), (16, 2, 64), (80, 4, 128), (1 << 24, 8, 128)):
        got = lib.slim_kv8_block_bytes(block, heads, d)
        assert got == ref.slot_bytes(block, heads, d) and got % 16 == 0
    for block, heads, d in ((0, 8, 128), (64, 0, 128), (64, 8, 32), (64, 8, 96), (64, 8, 256), (64, 8, 0), ((1 << 24) + 1, 8, 128), (64, 70000, 128)):
        assert lib.slim_kv8_block_bytes(block, heads, d) == 0


def batch_map(lib, lens=at(1 << 12), new=at(2 << 12), R=8, block=64, table=at(3 << 12), wide=10, free=at(4 << 12), n_free=50, used=at(5 << 12), slots=100, rows=64, lens_out=at(6 << 12),
              start=at(7 << 12), pos=at(8 << 12), slot=at(9 << 12), info=at(10 << 12)):
    return lib.slim_batch_map(lens, new, R, block, table, wide, free, n_free, used, slots, rows, lens_out, start, pos, slot, info, NULL)


def test_map_refusals(lib):
    for bad in (dict(lens=NULL), dict(new=NULL), dict(table=NULL), dict(free=NULL), dict(lens_out=NULL), dict(start=NULL), dict(pos=NULL), dict(slot=NULL), dict(info=NULL), dict(R=0),
                dict(block=0), dict(wide=0), dict(n_free=-1), dict(slots=0), dict(rows=0)):
        assert batch_map(lib, **bad) == -1, bad
    for bad in (dict(R=4097), dict(block=(1 << 24) + 1, wide=1), dict(block=1 << 20, wide=1025), dict(block=64, slots=1 << 25), dict(rows=1 << 29)):
        assert batch_map(lib, **bad) == -2, bad
    # what is written lies apart from everything else
    ins = dict(lens=(1 << 12, 32), new=(2 << 12, 32), free=(4 << 12, 200), used=(5 << 12, 4))
    outs = dict(table=(3 << 12, 320), lens_out=(6 << 12, 32), start=(7 << 12, 36), pos=(8 << 12, 256), slot=(9 << 12, 256), info=(10 << 12, 16))
    for name, (_, size) in outs.items():
        for other, (where, length) in {**ins, **outs}.items():
            if other != name:
                for x in (where, where + length - 4, where - size + 4):
                    assert batch_map(lib, **{name: at(x)}) == -1, (name, other, x)


def write(lib, k=ONE, v=ONE, ldk=1024, ldv=1024, places=ONE, n=100, heads=8, d=128, block=64, dtype=1, pool=ONE, slots=4, size=SIZE, off=0):
    return lib.slim_kv8_write(k, v, ldk, ldv, places, n, heads, d, block, dtype, pool, slots, size, off, NULL)


def read(lib, pool=ONE, slots=4, size=SIZE, off=0, lst=ONE, n=200, heads=8, d=128, block=64, dtype=1, k=ONE, v=ONE, ldk=1024, ldv=1024):
    return lib.slim_kv8_read(pool, slots, size, off, lst, n, heads, d, block, dtype, k, v, ldk, ldv, NULL)


POOL_INVALID = (dict(pool=NULL), dict(slots=0), dict(block=0), dict(heads=0), dict(d=0), dict(size=SIZE - 16), dict(off=16), dict(off=1 << 40), dict(k=NULL), dict(v=NULL), dict(ldk=1016),
                dict(ldv=1016), dict(n=0))
POOL_UNSUPPORTED = (dict(dtype=2), dict(d=96), dict(d=32), dict(heads=1, d=256), dict(heads=70000, ldk=1 << 24, ldv=1 << 24, size=1 << 60), dict(size=SIZE + 8), dict(size=SIZE + 16, off=8),
                    dict(pool=ODD), dict(k=ODD), dict(v=ODD), dict(ldk=1028), dict(ldv=1028), dict(dtype=0, ldk=1026), dict(block=(1 << 24) + 1, size=1 << 60),
                    dict(slots=1 << 25), dict(n=1 << 26), dict(n=1 << 29))


def test_write_and_read_refusals(lib):
    for call in (write, read):
        for bad in POOL_INVALID:
            assert call(lib, **bad) == -1, bad
        for bad in POOL_UNSUPPORTED:
            assert call(lib, **bad) == -2, bad
    assert write(lib, places=NULL) == -1


def attn(lib, q=ONE, ldq=4096, start=ONE, lens=ONE, table=ONE, R=3, n=5, wide=10, pool=ONE, slots=4, size=SIZE, off=0, block=64, Hq=32, heads=8, d=128, scale=0.0, dtype=1, out=ONE, ldo=4096,
         ws=ONE, ws_bytes=1 << 40):
    return lib.slim_batch_attn_kv8(q, ldq, start, lens, table, R, n, wide, pool, slots, size, off, block, Hq, heads, d, scale, dtype, out, ldo, ws, ws_bytes, NULL)


def test_attention_refusals(lib):
    for bad in (dict(q=NULL), dict(start=NULL), dict(lens=NULL), dict(table=NULL), dict(out=NULL), dict(ws=NULL), dict(pool=NULL), dict(R=0), dict(n=0), dict(wide=0), dict(slots=0),
                dict(block=0), dict(Hq=0), dict(heads=0), dict(Hq=33), dict(d=0), dict(size=SIZE - 16), dict(off=16), dict(scale=-1.0), dict(scale=float("nan")), dict(ldq=4088),
                dict(ldo=4088)):
        assert attn(lib, **bad) == -1, bad
    for bad in (dict(dtype=2), dict(d=96), dict(R=4097), dict(n=1 << 22, ldq=4096), dict(wide=1 << 25), dict(q=ODD), dict(out=ODD), dict(pool=ODD), dict(ws=at(128)), dict(ldq=4100),
                dict(ldo=4100), dict(slots=1 << 25), dict(R=4096, Hq=2048, heads=2048, ldq=1 << 18, ldo=1 << 18, size=1 << 40),
                dict(Hq=1 << 15, heads=1, ldq=1 << 22, ldo=1 << 22)):
        assert attn(lib, **bad) == -2, bad
    need = lib.slim_batch_attn_kv8_workspace_bytes(5, 3, 32, 8, 128)
    assert need > 0 and need % 256 == 0 and attn(lib, ws_bytes=need - 1) == -3
    for bad in ((0, 3, 32, 8, 128), (5, 0, 32, 8, 128), (5, 3, 0, 8, 128), (5, 3, 32, 0, 128), (5, 3, 33, 8, 128), (5, 3, 32, 8, 96), (5, 4097, 32, 8, 128), (1 << 22, 3, 32, 8, 128), (5, 3, 1 << 15, 1, 128)):
        assert lib.slim_batch_attn_kv8_workspace_bytes(*bad) == 0
    # a workspace for more rows serves fewer
    sizes = [lib.slim_batch_attn_kv8_workspace_bytes(n, 4, 32, 8, 128) for n in (1, 2, 64, 65, 1000, 100000)]
    assert sizes == sorted(sizes)


# --------------------------------------------------------------------------- what the binding refuses before it looks for a GPU (the tensors lie on the host)
def test_binding_refusals(slim):
    i = lambda *shape: torch.zeros(*shape, dtype=I32)
    with pytest.raises(ValueError, match="block_table"):
        slim.slim_batch_map(i(3), i(3), 16, i(2, 5), i(9), 20, 8)
    with pytest.raises(ValueError, match="block_table"):
        slim.slim_batch_map(i(3), i(3), 16, i(15), i(9), 20, 8)
    k = torch.zeros(8, 2, 64, dtype=BF16)
    pool = torch.zeros(2, slim.kv8_block_bytes(16, 2, 64), dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        slim.slim_kv8_write(k, k, pool, 16, i(8))
    with pytest.raises(ValueError, match="shorter"):
        slim.slim_kv8_read(pool, 16, 33, i(2), n_kv_heads=2, head_dim=64)
    with pytest.raises(ValueError, match="GPU"):
        slim.slim_kv8_read(pool, 16, 16, i(2), n_kv_heads=2, head_dim=64)
    with pytest.raises(ValueError, match="together"):
        slim.slim_kv8_read(pool, 16, 16, k_out=k)
    q = torch.zeros(5, 4, 64, dtype=BF16)
    with pytest.raises(ValueError, match="block_table"):
        slim.slim_batch_attn_kv8(q, i(4), i(3), i(2, 5), pool, 16, 2)
    for out in (torch.zeros(5, 2, 64, dtype=BF16), torch.zeros(5, 4, 64), torch.zeros(5, 4, 64, dtype=BF16)):
        with pytest.raises(ValueError, match="out"):
            slim.slim_batch_attn_kv8(q, i(4), i(3), i(3, 5), pool, 16, 2, out=out)
    with pytest.raises(ValueError, match="GPU"):
        slim.slim_batch_attn_kv8(q, i(4), i(3), i(3, 5), pool, 16, 2)


# ------------------------------------------------------------------------------------------------------------- the plain forms that the GPU's results are held to
def test_reference_codes_and_exponents():
    import numpy as np
    assert ref.GRID[1] == 2.0 ** -9 and ref.GRID[8] == 2.0 ** -6 and ref.GRID[126] == 448 and (np.diff(ref.GRID) > 0).all()
    assert (ref.codes(ref.GRID) == np.arange(127)).all() and (ref.codes(-ref.GRID) == 128 + np.arange(127)).all()
    mid = (ref.GRID[1:] + ref.GRID[:-1]) / 2
    assert (ref.codes(mid) % 2 == 0).all() and (ref.codes(mid * (1 + 2 ** -20)) == np.arange(1, 127)).all() and (ref.codes(mid * (1 - 2 ** -20)) == np.arange(126)).all()
    # torch's own e4m3, up to its largest value
    x = torch.randn(20000) * torch.exp2(torch.randint(-12, 9, (20000,)).float())
    x = x.clamp(-448, 448)
    assert (ref.codes(x.double().numpy()) == x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()).all()
    for e in (-117, -30, 0, 5, 119):
        top = 448 * 2.0 ** e
        got = ref.exponent(np.array([top, np.nextafter(np.float32(top), np.float32(0)), np.nextafter(np.float32(top), np.float32(1e38)), top / 2])) - 127
        assert got.tolist() == [e, e, min(e + 1, 119), max(e - 1, -117)]
    assert ref.exponent(np.array([0.0, 1e-45, 3.4e38])).tolist() == [10, 10, 246]
