"""Attention with a sliding window and visible first tokens on the GPU, against a plain implementation in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import kv4_reference as ref
from tests.test_gpu_kv4 import keys, rand

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def visible(n_q, n_k, window, sinks):
    p, j = np.arange(n_k - n_q, n_k)[:, None], np.arange(n_k)[None]
    return (j <= p) & ((j > p - window) | (j < sinks))


def inputs_of(n_q, n_k, Hq, Hkv, d, dtype, seed):
    return rand((n_q, Hq, d), dtype, seed, 0.6), keys(n_k, Hkv, d, dtype, seed + 1), rand((n_k, Hkv, d), dtype, seed + 2)


def check(got, q, k, v, window, sinks, scale=None, rows=None):
    """Against 64 bits, on some rows where there are many."""
    n_q, n_k, d = q.shape[0], k.shape[0], q.shape[2]
    rows = np.arange(n_q) if rows is None else rows
    seen = visible(n_q, n_k, window, sinks)[rows]
    want, size, reach = ref.attention(ref.to64(q)[rows], ref.to64(k), ref.to64(v), seen, scale or 1 / math.sqrt(d))
    ref.within(got[torch.from_numpy(rows).to(got.device)], want, ref.attention_bound(want, size, reach, int(seen.sum(1).max()), d, q.dtype, ref.to64(v)))


CASES = [
    # n_q, n_k, Hq, Hkv, d, window, sinks, dtype
    (1, 1, 1, 1, 128, 1, 0, BF16),
    (1, 1, 2, 1, 32, 1, 5, F32),
    (1, 700, 32, 8, 128, 100, 4, BF16),
    (1, 700, 28, 4, 128, 700, 0, F32),
    (1, 5000, 4, 2, 64, 3000, 33, F32),
    (1, 3100, 20, 1, 128, 3000, 64, BF16),            # 20 query heads per kv head
    (5, 333, 6, 2, 128, 1, 0, BF16),                  # a query sees itself alone
    (5, 333, 6, 2, 128, 1, 2, BF16),
    (17, 400, 10, 2, 128, 37, 40, BF16),
    (100, 100, 4, 2, 64, 33, 3, F32),
    (100, 100, 3, 3, 32, 1000, 0, F32),
    (64, 64, 4, 1, 128, 2**31 - 1, 2**31 - 1, BF16),
    (130, 517, 28, 4, 128, 129, 70, BF16),
    (300, 300, 8, 2, 128, 64, 0, BF16),
    (300, 300, 8, 2, 128, 64, 1, BF16),
    (517, 517, 5, 5, 128, 200, 130, BF16),
    (600, 700, 7, 1, 128, 31, 300, BF16),
    (257, 1000, 16, 2, 128, 1000, 0, BF16),
    (520, 520, 4, 1, 128, 520, 0, F32),
]


@pytest.mark.parametrize("n_q,n_k,Hq,Hkv,d,window,sinks,dtype", CASES)
def test_against_64_bits(slim, n_q, n_k, Hq, Hkv, d, window, sinks, dtype):
    print(f"sliding n_q={n_q} n_k={n_k} {Hq}/{Hkv} d={d} window={window} sinks={sinks} {dtype}", flush=True)
    q, k, v = inputs_of(n_q, n_k, Hq, Hkv, d, dtype, n_q + n_k)
    # what lies around the inputs and the output stays out and as it was
    room = torch.full((n_q + 2, Hq, d), 7.0, dtype=dtype, device="cuda")
    kk, vv = (torch.cat([torch.full_like(x[:3].repeat(3, 1, 1)[:3], math.nan), x, torch.full_like(x[:3].repeat(3, 1, 1)[:3], math.nan)]).cuda() for x in (k, v))
    out = slim.slim_sliding_attn(q.cuda(), kk[3:3 + n_k], vv[3:3 + n_k], window, sinks, out=room[1:1 + n_q])
    assert (room[0] == 7).all() and (room[-1] == 7).all()
    check(out, q, k, v, window, sinks, rows=np.unique(np.concatenate([np.arange(0, n_q, max(1, n_q // 40)), np.arange(max(0, n_q - 20), n_q), np.arange(min(n_q, 20))])))


@pytest.mark.parametrize("n_q,n_k,Hq,Hkv,d,window,sinks,dtype", [
    (1, 300, 4, 2, 128, 50, 3, BF16), (40, 300, 4, 2, 128, 50, 3, BF16), (40, 300, 4, 2, 64, 50, 3, F32), (300, 300, 8, 2, 128, 70, 10, BF16), (700, 700, 4, 1, 128, 130, 0, BF16),
    (600, 800, 3, 1, 128, 100, 40, BF16)])
def test_keys_and_values_that_a_query_does_not_see_do_not_reach_it(slim, n_q, n_k, Hq, Hkv, d, window, sinks, dtype):
    """Infinities and NaN in keys and values: the rows that do not see them are what they are without them."""
    q, k, v = inputs_of(n_q, n_k, Hq, Hkv, d, dtype, 11)
    places = sorted({0, sinks, n_k - n_q, n_k - 1, n_k // 2, max(0, n_k - n_q - window), max(0, n_k - window), n_k - n_q + n_q // 3} & set(range(n_k)))
    seen = visible(n_q, n_k, window, sinks)
    want, size, reach = ref.attention(ref.to64(q), ref.to64(k), ref.to64(v), seen, 1 / math.sqrt(d))
    bound = ref.attention_bound(want, size, reach, int(seen.sum(1).max()), d, dtype, ref.to64(v))
    for which in ("v", "k"):
        for value in (math.inf, math.nan):
            for bad in (places, places[::2], places[1::2], [places[-1]]):
                kk, vv = k.clone(), v.clone()
                (vv if which == "v" else kk)[bad] = value
                got = slim.slim_sliding_attn(q.cuda(), kk.cuda(), vv.cuda(), window, sinks)
                blind = ~seen[:, bad].any(1)
                print(which, value, bad, int(blind.sum()), end="", flush=True)
                if blind.any():
                    ref.within(got[torch.from_numpy(blind).cuda()], want[blind], bound[blind])
                if which == "v":
                    assert not torch.isfinite(got[torch.from_numpy(~blind).cuda()].float()).all(-1).any()


def test_window_that_covers_everything_is_plain_causal_attention(slim):
    n, Hq, Hkv, d = 900, 8, 2, 128
    q, k, v = inputs_of(n, n, Hq, Hkv, d, BF16, 5)
    out = slim.slim_sliding_attn(q.cuda(), k.cuda(), v.cuda(), n)
    full = slim.slim_prefill_attn(q.cuda(), k.cuda(), v.cuda())
    check(full, q, k, v, n, 0, rows=np.arange(0, n, 37))
    check(out, q, k, v, n, 0, rows=np.arange(0, n, 37))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (2, 0), (16, 4), (17, 0)])
def test_short_windows_of_many_queries(slim, window, sinks):
    """Most units of a tile of 256 rows hold nothing for most of its rows."""
    q, k, v = inputs_of(1100, 1133, 32, 8, 128, BF16, 12)
    out = slim.slim_sliding_attn(q.cuda(), k.cuda(), v.cuda(), window, sinks)
    check(out, q, k, v, window, sinks, rows=np.unique(np.concatenate((np.arange(0, 1100, 41), np.arange(1080, 1100)))))


@pytest.mark.parametrize("n_q,n_k,window,sinks", [(1100, 1100, 300, 1), (1100, 1100, 300, 32), (1100, 1100, 257, 33), (1100, 1133, 300, 96), (1100, 1133, 290, 97), (1100, 1133, 290, 200),
                                                  (512, 3000, 2000, 64), (512, 3001, 2001, 90), (512, 3000, 2000, 129), (480, 2100, 2000, 70)])
def test_first_tokens_of_many_queries(slim, n_q, n_k, window, sinks):
    """First tokens that share a tile with the window's beginning, that fill tiles, that meet it; the keys in one part and in several."""
    q, k, v = inputs_of(n_q, n_k, 32, 8, 128, BF16, 13)
    k[:sinks] *= 2                                        # what the first tokens hold counts
    out = slim.slim_sliding_attn(q.cuda(), k.cuda(), v.cuda(), window, sinks)
    check(out, q, k, v, window, sinks, rows=np.unique(np.concatenate((np.arange(0, n_q, 41), np.arange(n_q - 20, n_q)))))


def test_chunks_and_single_tokens_give_the_rows_of_the_whole(slim):
    n, Hq, Hkv, d, window, sinks = 300, 8, 2, 128, 77, 5
    q, k, v = (x.cuda() for x in inputs_of(n, n, Hq, Hkv, d, BF16, 6))
    whole = slim.slim_sliding_attn(q, k, v, window, sinks).double()
    for a, b in ((0, 1), (1, 2), (40, 41), (120, 140), (140, 290), (299, 300)):
        part = slim.slim_sliding_attn(q[a:b].contiguous(), k[:b], v[:b], window, sinks).double()
        # both are within half a bfloat16 step and the weights' rounding of the same numbers: 4 * 2^-8 of the values' size
        assert ((part - whole[a:b]).abs() <= 4 * 2.0 ** -8 * v[:b].double().abs().amax()).all()
        assert ((part - whole[a:b]).abs().mean() <= 2.0 ** -9)


def test_large_and_flat_scores(slim):
    n, H, d = 700, 2, 128
    for n_q in (1, 50, 700):
        k, v = torch.ones(n, H, d), rand((n, H, d), F32, 1)
        k[n // 2] = 9.0
        k[n // 3] = -9.0
        q = torch.zeros(n_q, 2 * H, d)
        q[:, 1], q[:, 2] = 5.0, -5.0                      # logits of +-500 (one key takes everything) and flat ones
        for dtype in (BF16, F32):
            x = [t.to(dtype) for t in (q, k, v)]
            out = slim.slim_sliding_attn(*(t.cuda() for t in x), 400, 7)
            check(out, *x, 400, 7, rows=np.unique(np.linspace(0, n_q - 1, 30).astype(int)))


def test_scale(slim):
    q, k, v = inputs_of(20, 90, 4, 2, 128, BF16, 8)
    out = slim.slim_sliding_attn(q.cuda(), k.cuda(), v.cuda(), 50, 2, softmax_scale=0.3)
    check(out, q, k, v, 50, 2, scale=float(np.float32(0.3)))


def test_binding_refusals(slim):
    q, k = torch.zeros(4, 4, 128, dtype=BF16, device="cuda"), torch.zeros(9, 2, 128, dtype=BF16, device="cuda")
    for bad in (lambda: slim.slim_sliding_attn(q, k, k[:8], 4), lambda: slim.slim_sliding_attn(q, k, k.float(), 4), lambda: slim.slim_sliding_attn(q, k[:, :, :64], k[:, :, :64], 4),
                lambda: slim.slim_sliding_attn(q, k, k, 4, out=q[:3]), lambda: slim.slim_sliding_attn(q.cpu(), k, k, 4), lambda: slim.slim_sliding_attn(q.transpose(0, 1), k, k, 4)):
        with pytest.raises(ValueError):
            bad()
    for bad in (dict(window=0), dict(window=4, n_sinks=-1), dict(window=4, softmax_scale=-1.0)):
        with pytest.raises(slim.SlimError):
            slim.slim_sliding_attn(q, k, k, **bad)
    with pytest.raises(slim.SlimError):
        slim.slim_sliding_attn(torch.zeros(10, 4, 128, dtype=BF16, device="cuda"), k, k, 4)             # more queries than keys


def test_workspace_is_written_within_its_bounds_and_its_contents_do_not_matter(slim):
    q, k, v = (x.cuda() for x in inputs_of(3, 3000, 8, 2, 128, BF16, 9))
    need = slim.sliding_attn_workspace_bytes(3, 3000, 8, 2, 128, 2000, 64, BF16)
    assert need > 0
    outs = []
    for fill in (0, 255):
        ws = torch.full((need + 4096,), fill, dtype=torch.uint8, device="cuda")
        outs.append(slim.slim_sliding_attn(q, k, v, 2000, 64, workspace=ws[:need]))
        assert (ws[need:] == fill).all()
    assert torch.equal(*outs)


def test_replayed_from_a_graph(slim):
    shapes = [(1, 3000, 32, 8, 128, 1024, 64, BF16), (700, 900, 8, 2, 128, 200, 10, BF16), (50, 300, 4, 2, 64, 70, 3, F32)]
    state = []
    for s in shapes:
        q, k, v = (x.cuda() for x in inputs_of(*s[:5], s[7], 3))
        state.append((q, k, v, torch.zeros_like(q), torch.empty(max(256, slim.sliding_attn_workspace_bytes(*s)), dtype=torch.uint8, device="cuda"), s[5], s[6]))

    def step():
        for q, k, v, out, ws, window, sinks in state:
            slim.slim_sliding_attn(q, k, v, window, sinks, out=out, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    for seed in range(3):
        for q, k, *_ in state:
            q.copy_(rand(q.shape, q.dtype, 30 + seed))
            k.copy_(keys(*k.shape, k.dtype, 40 + seed))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [st[3].clone() for st in state]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, st[3]) for a, st in zip(got, state))
