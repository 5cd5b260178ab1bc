"""Sliding-window attention in tiles of 256 rows (bfloat16, many queries), where it can go wrong, on calls that take this kernel: with a row tile's keys in one part and in several.

What a call takes is a rule on sizes (csrc/sliding_plan.h); test_the_shapes_take_the_kernel holds the shapes to it without a GPU."""
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from tests import kv4_reference as ref
from tests.test_gpu_kv4 import BF16, F32, keys, rand
from tests.test_gpu_sliding import inputs_of, visible

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# n_q, n_k, Hq, Hkv, window, first tokens, parts of a row tile's keys
ONE = [
    (1100, 1133, 32, 8, 290, 0, 1),
    (1100, 1133, 32, 8, 290, 40, 1),
    (3000, 3000, 28, 4, 130, 0, 1),                      # 7 query heads per kv head
    (1000, 1200, 24, 8, 40, 9, 1),                       # 3
    (700, 700, 24, 8, 700, 0, 1),
    (700, 900, 40, 8, 200, 150, 1),                      # 5, first tokens that fill a tile of their own
    (800, 1000, 56, 8, 150, 33, 1),
    (500, 500, 20, 1, 500, 3, 1),                        # 20
    (2000, 2000, 16, 16, 64, 0, 1),                      # 1
]
PARTS = [
    (900, 900, 8, 2, 900, 0, 4),
    (512, 3000, 32, 8, 2000, 64, 3),
    (600, 3000, 28, 4, 2900, 0, 3),
    (500, 1500, 20, 1, 1500, 3, 4),
    (450, 2100, 18, 6, 2000, 130, 6),
]
LARGE = (2200, 2200, 32, 8, 2200, 0, 1)                  # many tiles without a mask


def test_the_shapes_take_the_kernel(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no host compiler")
    shapes = ONE + PARTS + [LARGE]
    calls = "".join(f'    printf("%d\\n", sliding_parts({m}, {n}, {Hq // Hkv}, {Hkv}, {min(w, n)}, {min(s, n)}));\n' for m, n, Hq, Hkv, w, s, _ in shapes)
    src, exe = tmp_path / "routes.cpp", tmp_path / "routes"
    src.write_text('#include "sliding_plan.h"\n#include <cstdio>\nusing namespace slim;\nint main() {\n' + calls + "}\n")
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2508_06447_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [s[-1] for s in shapes]


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def attention64(q, k, v, seen, scale):
    """ref.attention's three results, in float64 on the GPU, head by head; seen[m, n] on the host."""
    m, Hq, d = q.shape
    G, seen = Hq // k.shape[1], torch.from_numpy(seen).cuda()
    out, size = (torch.empty(m, Hq, d, dtype=torch.float64, device="cuda") for _ in range(2))
    reach = 0.0
    for h in range(Hq):
        qq, kk, vv = (x.cuda().double().contiguous() for x in (q[:, h], k[:, h // G], v[:, h // G]))
        p = torch.softmax((torch.mm(qq, kk.t().contiguous()) * scale).masked_fill_(~seen, -math.inf), -1)
        out[:, h], size[:, h] = torch.mm(p, vv), torch.mm(p, vv.abs())
        reach = max(reach, float((torch.mm(qq.abs(), kk.abs().t().contiguous()) * seen).max()) * scale)
    return out.cpu().numpy(), size.cpu().numpy(), reach


def answer(q, k, v, window, sinks, scale=None):
    """(result, bound, what each query sees)."""
    d = q.shape[2]
    seen = visible(q.shape[0], k.shape[0], window, sinks)
    want, size, reach = attention64(q, k, v, seen, scale or 1 / math.sqrt(d))
    return want, ref.attention_bound(want, size, reach, int(seen.sum(1).max()), d, q.dtype, ref.to64(v)), seen


def need_of(slim, n_q, n_k, Hq, Hkv, window, sinks, parts):
    need = slim.sliding_attn_workspace_bytes(n_q, n_k, Hq, Hkv, 128, window, sinks, BF16)
    assert need == (-(-parts * n_q * Hq * 132 * 4 // 256) * 256 if parts > 1 else 0)              # rows of 132 floats
    return need


@pytest.mark.gpu
@pytest.mark.parametrize("shape", ONE + PARTS + [LARGE])
def test_against_64_bits(slim, shape):
    """Results, and what lies around inputs, outputs and partial results; a workspace's contents do not matter."""
    n_q, n_k, Hq, Hkv, window, sinks, parts = shape
    print(f"many {shape}", flush=True)
    q, k, v = inputs_of(n_q, n_k, Hq, Hkv, 128, BF16, n_q + n_k)
    if sinks:
        k[:sinks] *= 2
    want, bound, _ = answer(q, k, v, window, sinks)
    need = need_of(slim, *shape)
    room = torch.full((n_q + 2, Hq, 128), 7.0, dtype=BF16, device="cuda")
    edge = torch.full((3, Hkv, 128), math.nan, dtype=BF16)
    kk, vv = (torch.cat([edge, x, edge]).cuda() for x in (k, v))
    outs = []
    for fill in (0, 255):
        ws = torch.full((need + 4096,), fill, dtype=torch.uint8, device="cuda")
        out = slim.slim_sliding_attn(q.cuda(), kk[3:3 + n_k], vv[3:3 + n_k], window, sinks, out=room[1:1 + n_q], workspace=ws[:need] if need else None)
        assert (room[0] == 7).all() and (room[-1] == 7).all() and (ws[need:] == fill).all()
        outs.append(out.clone())
    assert torch.equal(*outs)
    ref.within(outs[0], want, bound)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [ONE[0], ONE[1], ONE[3], ONE[5], ONE[7], PARTS[0], PARTS[1], PARTS[4]])
def test_what_a_query_does_not_see_does_not_reach_it(slim, shape):
    """Infinities and NaN in keys and values: the rows that do not see them are what they are without them, the ones that see such a value are not finite."""
    n_q, n_k, Hq, Hkv, window, sinks, parts = shape
    q, k, v = inputs_of(n_q, n_k, Hq, Hkv, 128, BF16, 11)
    want, bound, seen = answer(q, k, v, window, sinks)
    first = n_k - n_q
    places = sorted({0, sinks, first, n_k - 1, n_k // 2, max(0, first - window), max(0, first - window + 1), max(0, n_k - window), first + n_q // 3} & set(range(n_k)))
    for which in ("v", "k"):
        for value in (math.inf, -math.inf, math.nan):
            for bad in (places, places[1::2], [places[-1]], [places[-2]]):
                kk, vv = k.clone(), v.clone()
                (vv if which == "v" else kk)[bad] = value
                got = slim.slim_sliding_attn(q.cuda(), kk.cuda(), vv.cuda(), window, sinks)
                blind = ~seen[:, bad].any(1)
                print(shape, which, value, bad, int(blind.sum()), end="", flush=True)
                if blind.any():
                    ref.within(got[torch.from_numpy(blind).cuda()], want[blind], bound[blind])
                if which == "v":
                    assert not torch.isfinite(got[torch.from_numpy(~blind).cuda()].float()).all(-1).any()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [LARGE, ONE[0], ONE[5], ONE[6], PARTS[0], PARTS[1], PARTS[2]])
@pytest.mark.parametrize("towers", ["rising", "one late", "one early", "falling"])
def test_logits_far_apart(slim, shape, towers):
    """A reference that the logits leave by far more than a float's exponent: keys that tower over the others in every unit of a tile, and in tiles with and without masks."""
    n_q, n_k, Hq, Hkv, window, sinks, parts = shape
    need_of(slim, *shape)
    q, k, v = torch.zeros(n_q, Hq, 128), torch.zeros(n_k, Hkv, 128), rand((n_k, Hkv, 128), F32, 1)
    # logits 8 * k[0] / sqrt(128), and small ones in the other channels
    q[:, :, 0] = 8.0
    q[:, :, 1:] = rand((n_q, Hq, 127), F32, 2, 0.2)
    k[:, :, 1:] = rand((n_k, Hkv, 127), F32, 3, 0.2)
    at = np.arange(5, n_k, 37)                            # 37 keys apart: every unit of 32 in turn
    if towers == "rising":
        k[at, :, 0] = torch.from_numpy(80.0 * np.arange(1, len(at) + 1) / max(1, len(at) / 12)).float()[:, None]
    elif towers == "falling":
        k[at, :, 0] = torch.from_numpy(80.0 * np.arange(len(at), 0, -1) / max(1, len(at) / 12)).float()[:, None]
    else:
        k[n_k - 7 if towers == "one late" else 1, :, 0] = 700.0      # logits of 500
        k[n_k // 2, :, 0] = -700.0
    q, k, v = (x.to(BF16) for x in (q, k, v))
    want, bound, _ = answer(q, k, v, window, sinks)
    ref.within(slim.slim_sliding_attn(q.cuda(), k.cuda(), v.cuda(), window, sinks), want, bound)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [ONE[1], ONE[2], PARTS[0], PARTS[1]])
@pytest.mark.parametrize("scale", [0.3, 2.0 ** -10])
def test_scale(slim, shape, scale):
    n_q, n_k, Hq, Hkv, window, sinks, parts = shape
    q, k, v = inputs_of(n_q, n_k, Hq, Hkv, 128, BF16, 8)
    want, bound, _ = answer(q, k, v, window, sinks, float(np.float32(scale)))
    ref.within(slim.slim_sliding_attn(q.cuda(), k.cuda(), v.cuda(), window, sinks, softmax_scale=scale), want, bound)


def state_of(slim, shape, seed):
    n_q, n_k, Hq, Hkv, window, sinks, parts = shape
    q, k, v = (x.cuda() for x in inputs_of(n_q, n_k, Hq, Hkv, 128, BF16, seed))
    need = need_of(slim, *shape)
    return q, k, v, torch.zeros_like(q), torch.empty(need, dtype=torch.uint8, device="cuda") if need else None, window, sinks


def call(slim, st):
    q, k, v, out, ws, window, sinks = st
    return slim.slim_sliding_attn(q, k, v, window, sinks, out=out, workspace=ws)


@pytest.mark.gpu
def test_replayed_from_a_graph(slim):
    state = [state_of(slim, s, 3) for s in (ONE[1], ONE[7], PARTS[0], PARTS[1])]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for st in state:
            call(slim, st)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            for st in state:
                call(slim, st)
    for seed in range(3):
        for q, k, *_ in state:
            q.copy_(rand(q.shape, q.dtype, 30 + seed))
            k.copy_(keys(*k.shape, k.dtype, 40 + seed))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [st[3].clone() for st in state]
        for st, x in zip(state, got):
            st[3].zero_()
            assert torch.equal(call(slim, st), x)


@pytest.mark.gpu
def test_two_calls_at_once(slim):
    """On streams of their own, with workspaces of their own."""
    state = [state_of(slim, s, 5 + i) for i, s in enumerate((PARTS[1], PARTS[0]))]
    alone = [call(slim, st).clone() for st in state]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in state]
    for _ in range(5):
        for st, s in zip(state, streams):
            st[3].zero_()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                call(slim, st)
        torch.cuda.synchronize()
        assert all(torch.equal(st[3], x) for st, x in zip(state, alone))


@pytest.mark.gpu
@pytest.mark.parametrize("n_q,n_k,Hq,Hkv,dtype", [(1, 3000, 32, 8, BF16), (900, 900, 8, 2, BF16), (40, 300, 4, 2, F32)])
def test_windows_and_first_tokens_beyond_32_bits(slim, n_q, n_k, Hq, Hkv, dtype):
    """Beyond the keys, all of them are meant: however far beyond."""
    import sys
    q, k, v = (x.cuda() for x in inputs_of(n_q, n_k, Hq, Hkv, 128, dtype, 4))
    whole = slim.slim_sliding_attn(q, k, v, n_k)
    size = slim.sliding_attn_workspace_bytes(n_q, n_k, Hq, Hkv, 128, n_k, 0, dtype)
    for far in (2**31, 2**32 + 3, 2**32, 2**40 + 1, sys.maxsize):
        assert torch.equal(slim.slim_sliding_attn(q, k, v, far), whole)
        assert slim.sliding_attn_workspace_bytes(n_q, n_k, Hq, Hkv, 128, far, 0, dtype) == size
        assert torch.equal(slim.slim_sliding_attn(q, k, v, 5, far), slim.slim_sliding_attn(q, k, v, 5, n_k))
    for none in (0, -1, -2**32 + 3, -sys.maxsize):
        with pytest.raises(slim.SlimError):
            slim.slim_sliding_attn(q, k, v, none)
