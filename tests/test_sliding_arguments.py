"""Sliding-window attention: workspaces and what is refused before anything is enqueued (no GPU)."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2508_06447_amd as slim
    if not os.path.exists(slim.LIB_PATH):
        from paper_2508_06447_amd.build import build_lib
        build_lib(verbose=False)
    return slim.load_library()


NULL, ONE = ctypes.c_void_p(0), ctypes.c_void_p(256)      # the second: never dereferenced on these paths


def call(lib, q=ONE, k=ONE, v=ONE, n_q=1, n_k=4096, Hq=32, Hkv=8, d=128, window=1024, sinks=4, scale=0.0, dtype=1, out=ONE, ws=ONE, wb=1 << 30):
    return lib.slim_sliding_attn(q, k, v, n_q, n_k, Hq, Hkv, d, window, sinks, ctypes.c_float(scale), dtype, out, ws, wb, NULL)


def test_refusals(lib):
    for bad in (dict(q=NULL), dict(k=NULL), dict(v=NULL), dict(out=NULL), dict(n_q=0), dict(n_q=4097), dict(Hq=30), dict(Hq=0), dict(Hkv=0), dict(d=0), dict(window=0),
                dict(window=-5), dict(sinks=-1), dict(scale=-0.5), dict(scale=float("nan")), dict(ws=NULL)):
        assert call(lib, **bad) == -1, bad
    for bad in (dict(dtype=2), dict(d=64), dict(d=96, dtype=0), dict(q=ctypes.c_void_p(264)), dict(out=ctypes.c_void_p(258)), dict(ws=ctypes.c_void_p(272)), dict(n_k=(1 << 30) + 1),
                dict(Hkv=70000, Hq=70000), dict(n_q=1 << 26, n_k=1 << 26),
                dict(n_q=(1 << 22) + 1, n_k=1 << 23), dict(n_q=(1 << 27) + 1, n_k=1 << 28, Hq=1, Hkv=1, d=32, dtype=0)):
        assert call(lib, **bad) == -2, bad
    assert call(lib, wb=16) == -3


def test_workspaces(lib):
    size = lib.slim_sliding_attn_workspace_bytes
    assert size(1, 4096, 32, 8, 128, 1024, 4, 1) > 0 and size(1, 4096, 32, 8, 128, 1024, 4, 1) % 256 == 0
    assert size(4096, 4096, 32, 8, 128, 1024, 4, 1) == 0                # many rows: none
    assert size(1, 1, 1, 1, 32, 1, 0, 0) == 0                           # one key: none
    for bad in ((0, 4, 4, 2, 128, 4, 0, 1), (5, 4, 4, 2, 128, 4, 0, 1), (1, 4, 3, 2, 128, 4, 0, 1), (1, 4, 4, 2, 64, 4, 0, 1), (1, 4, 4, 2, 128, 0, 0, 1), (1, 4, 4, 2, 128, 4, -1, 1),
                (1, 4, 4, 2, 128, 4, 0, 5)):
        assert size(*bad) == 0, bad
    assert call(lib, wb=size(1, 4096, 32, 8, 128, 1024, 4, 1) - 1) == -3
