"""The calls on a cache in 4 bits: sizes, and what is refused before anything is enqueued (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from tests import kv4_reference as ref


@pytest.fixture(scope="module")
def lib():
    import os

    import paper_2508_06447_amd as slim
    if not os.path.exists(slim.LIB_PATH):
        from paper_2508_06447_amd.build import build_lib
        build_lib(verbose=False)
    return slim.load_library()


NULL, ONE = ctypes.c_void_p(0), ctypes.c_void_p(256)      # the second: never dereferenced on these paths


def test_block_bytes(lib):
    assert lib.slim_kv4_block_bytes(64, 8, 128) == 64 * 8 * 136 == ref.slot_bytes(64, 8, 128)
    for block, heads, d in ((1, 1, 32), (7, 3, 64), (16, 2, 64), (80, 4, 128), (1 << 24, 8, 128)):
        got = lib.slim_kv4_block_bytes(block, heads, d)
        assert got == ref.slot_bytes(block, heads, d) and got % 16 == 0
    for block, heads, d in ((0, 8, 128), (64, 0, 128), (64, 8, 96), (64, 8, 256), (64, 8, 0), ((1 << 24) + 1, 8, 128), (64, 70000, 128)):
        assert lib.slim_kv4_block_bytes(block, heads, d) == 0


def write(lib, k=ONE, v=ONE, ldk=1024, ldv=1024, first=0, n=100, heads=8, d=128, block=64, dtype=1, sob=ONE, nb=8, pool=ONE, slots=4, size=64 * 8 * 136, at=0):
    return lib.slim_kv4_write(k, v, ldk, ldv, first, n, heads, d, block, dtype, sob, nb, pool, slots, size, at, NULL)


def read(lib, pool=ONE, slots=4, size=64 * 8 * 136, at=0, sob=ONE, blocks=ONE, n_list=2, block=64, n=500, heads=8, d=128, dtype=1, k=ONE, v=ONE, rows=128, ldk=1024, ldv=1024):
    return lib.slim_kv4_read(pool, slots, size, at, sob, blocks, n_list, block, n, heads, d, dtype, k, v, rows, ldk, ldv, NULL)


def test_write_refusals(lib):
    for bad in (dict(k=NULL), dict(v=NULL), dict(pool=NULL), dict(ldk=1016), dict(ldv=1016), dict(first=-1), dict(n=0), dict(heads=0), dict(d=0), dict(block=0), dict(nb=0),
                dict(slots=0), dict(n=513), dict(first=413), dict(size=64 * 8 * 136 - 16), dict(at=16), dict(at=1 << 40), dict(first=2**31 - 1, n=2**31 - 1)):
        assert write(lib, **bad) == -1, bad
    for bad in (dict(dtype=2), dict(d=96, ldk=4096, ldv=4096), dict(heads=1, d=256), dict(size=64 * 8 * 136 + 8), dict(size=64 * 8 * 136 + 64, at=8), dict(k=ctypes.c_void_p(264)),
                dict(pool=ctypes.c_void_p(264)), dict(ldk=1028), dict(ldv=1028), dict(dtype=0, ldk=1026), dict(block=(1 << 24) + 1, size=1 << 60), dict(n=1 << 29, nb=1 << 24),
                dict(first=(1 << 31) - 70000, n=10000, nb=1 << 26)):
        assert write(lib, **bad) == -2, bad


def test_read_refusals(lib):
    for bad in (dict(k=NULL), dict(v=NULL), dict(pool=NULL), dict(ldk=1016), dict(n=0), dict(n_list=0), dict(n_list=9), dict(rows=0), dict(heads=0), dict(block=0), dict(slots=0),
                dict(size=64 * 8 * 136 - 16), dict(at=16)):
        assert read(lib, **bad) == -1, bad
    for bad in (dict(dtype=7), dict(d=48, ldk=4096, ldv=4096), dict(size=64 * 8 * 136 + 8), dict(v=ctypes.c_void_p(257)), dict(ldv=1028), dict(n=1 << 29)):
        assert read(lib, **bad) == -2, bad


def attn(lib, q=ONE, pool=ONE, size=64 * 8 * 136, at=0, bos=ONE, slots=128, block=64, n=30000, kr=NULL, vr=NULL, nr=0, Hq=32, Hkv=8, d=128, scale=0.0, dtype=1, out=ONE, ws=ONE,
         wb=1 << 30):
    return lib.slim_decode_attn_kv4(q, pool, size, at, bos, slots, block, n, kr, vr, nr, Hq, Hkv, d, ctypes.c_float(scale), dtype, out, ws, wb, NULL)


def test_attention_refusals(lib):
    for bad in (dict(q=NULL), dict(out=NULL), dict(ws=NULL), dict(pool=NULL), dict(bos=NULL), dict(slots=-1), dict(slots=0), dict(nr=-1), dict(nr=3), dict(Hq=30), dict(Hq=0),
                dict(Hkv=0), dict(block=0), dict(n=0), dict(size=64 * 8 * 136 - 16), dict(at=16), dict(scale=-1.0), dict(scale=float("nan"))):
        assert attn(lib, **bad) == -1, bad
    for bad in (dict(dtype=3), dict(d=64), dict(Hq=136, Hkv=8), dict(size=64 * 8 * 136 + 8), dict(q=ctypes.c_void_p(264)), dict(ws=ctypes.c_void_p(272)),
                dict(kr=ctypes.c_void_p(264), vr=ONE, nr=1), dict(n=2**31 - 1), dict(slots=2**30, block=64)):
        assert attn(lib, **bad) == -2, bad
    assert attn(lib, wb=16) == -3
    assert attn(lib, wb=lib.slim_decode_attn_workspace_bytes(128, 0, 32) - 1) == -3


def test_layer_refusals(lib):
    import paper_2508_06447_amd as slim
    shape = slim.make_shape(4096, 32, 8, 128, 14336, 64, 8, 64, torch.bfloat16)
    w = slim.LayerWeights(*([256] * 9))
    call = lambda size, ws=1 << 30, s=shape: lib.slim_decode_layer_kv4(ctypes.byref(s), ctypes.byref(w), ONE, 40000, ONE, size, 0, ONE, 128, 30000, ONE, ONE, 3, ONE, NULL,
                                                                       ONE, ws, NULL)
    assert call(64 * 8 * 136 - 16) == -1 and call(64 * 8 * 136, 4096) == -3
    assert call(64 * 8 * 136, s=slim.make_shape(4096, 136, 8, 128, 14336, 64, 8, 64, torch.bfloat16)) == -2        # 17 query heads per kv head


def test_the_reference_rounds_as_stated():
    x = np.zeros((3, 32))
    x[0, :9] = (6.9, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.1)
    x[1, :2] = (7.0, 3.4)                                # one step further: e = 1
    x[2, 0] = np.inf
    code, byte = ref.quantise(x)
    assert code[0, :9].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 15] and byte[:, 0].tolist() == [127, 128, 255]
    assert code[1, :2].tolist() == [6, 3]
    got = ref.values(code, byte)
    assert got[1, 0] == 8.0 and got[1, 1] == 3.0 and np.isnan(got[2]).all()
    g = np.random.default_rng(0).standard_normal((100, 64)) * np.exp2(np.random.default_rng(1).integers(-20, 20, (100, 1)))
    back = ref.cached(g)
    most = np.abs(g.reshape(100, 2, 32)).max(-1).repeat(32, -1).reshape(100, 64)
    assert (np.abs(back - g) <= most / 3.5).all() and (ref.cached(back) == back).mean() > 0.99   # half of the largest step, which is 2 * 2^e <= 2 / 3.5 of the magnitude
