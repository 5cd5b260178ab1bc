"""A cache in 4 bits as it is used: the decoded token's layer over it, and a run of writing, choosing, swapping, attending, reading back and a follow-up prompt, against 64 bits."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import slim_oracle as so
from paper_2508_06447_amd import inputs
from tests import kv4_reference as ref
from tests.helpers import errs, f64
from tests.test_gpu_kv4 import keys, pool_of, rand

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def layer_case(slim, wl, dtype, n_slots, n_active, n_resp, fold, seed):
    """One decoded token through slim_decode_layer_kv4 against the oracle's layer on the values that the cache holds."""
    Hq, Hkv, d, block, n = wl.n_q_heads, wl.n_kv_heads, wl.head_dim, wl.block, wl.seq
    g = np.random.default_rng(seed)
    w = {k: v.to(dtype) for k, v in inputs.layer_weights(wl).items()}
    k, v = rand((n, Hkv, d), dtype, seed + 1), rand((n, Hkv, d), dtype, seed + 2)
    nb = -(-n // block)
    order = np.full(n_slots, -1, np.int32)
    active = np.concatenate([g.permutation(nb - 1)[:n_active - 1], [nb - 1]])
    order[g.permutation(n_slots)[:n_active]] = active
    pool = pool_of(slim, k, v, block, n_slots, order, seed)
    kr, vr = torch.zeros(n_resp + 1, Hkv, d, dtype=dtype), torch.zeros(n_resp + 1, Hkv, d, dtype=dtype)
    kr[:n_resp], vr[:n_resp] = rand((n_resp, Hkv, d), dtype, seed + 4), rand((n_resp, Hkv, d), dtype, seed + 5)
    x = rand((wl.hidden,), dtype, seed + 6, 1.5)
    shape = slim.make_shape(wl.hidden, Hq, Hkv, d, wl.ffn, block, wl.unit, wl.window, dtype, wl.rope_theta, wl.rms_eps)
    wd = {kk: vv.cuda() for kk, vv in w.items() if not (fold and kk in ("g_attn", "g_ffn"))}
    krd, vrd = kr.cuda(), vr.cuda()
    z, q = slim.slim_decode_layer_kv4(shape, wd, x.cuda(), n + n_resp, pool, torch.from_numpy(order).cuda(), n, krd, vrd, n_resp)
    s = so.LayerShape(wl.hidden, Hq, Hkv, d, wl.ffn, block, wl.unit, wl.window, wl.rope_theta, wl.rms_eps)
    ow = so.LayerWeights(**{kk: f64(vv) for kk, vv in w.items()})
    T = so.active_token_index(set(active.tolist()), block, n)
    k_ctx = np.concatenate([ref.cached(f64(k))[T], f64(kr[:n_resp])])
    v_ctx = np.concatenate([ref.cached(f64(v))[T], f64(vr[:n_resp])])
    z_ref, k_ref, v_ref = so.decode_layer(s, ow, f64(x), n + n_resp, k_ctx, v_ctx)
    mx, mean = errs(z, z_ref)
    print(f"kv4 layer {wl.family} {dtype} hidden {wl.hidden} slots {n_slots} resp {n_resp} fold {fold}: z max-abs {mx:.3e} mean-abs {mean:.3e}", flush=True)
    if dtype == BF16:
        z_b, _, _ = so.decode_layer(s, ow, f64(x), n + n_resp, k_ctx, v_ctx, rounding="bf16")
        assert mx <= max(2e-2, 1.5 * np.abs(z_b - z_ref).max()) and mean <= max(2e-3, 1.5 * np.abs(z_b - z_ref).mean())
    else:
        assert mx <= 2e-4                                # the parity bar of float32 layers
    rel = 2.0 ** -8 if dtype == BF16 else 1e-5
    np.testing.assert_allclose(f64(krd[n_resp]), k_ref, rtol=rel, atol=rel * np.abs(k_ref).max())
    np.testing.assert_allclose(f64(vrd[n_resp]), v_ref, rtol=rel, atol=rel * np.abs(v_ref).max())
    assert torch.equal(krd[:n_resp].cpu(), kr[:n_resp]) and torch.equal(vrd[:n_resp].cpu(), vr[:n_resp])


@pytest.mark.parametrize("fold", [False, True])
def test_decode_layer(slim, fold):
    llama = inputs.scaled(inputs.WORKLOADS["cfg2"], seq=1000, hidden=512, n_q_heads=8, n_kv_heads=2, ffn=1024)
    layer_case(slim, llama, BF16, 12, 9, 5, fold, 50)
    layer_case(slim, llama, BF16, 4, 4, 0, fold, 60)
    qwen = inputs.scaled(inputs.WORKLOADS["cfg6"], seq=777, hidden=448, n_q_heads=14, n_kv_heads=2, ffn=1184, x_kind="normal")
    layer_case(slim, qwen, BF16, 10, 7, 70, fold, 70)
    layer_case(slim, inputs.scaled(llama, n_q_heads=16, n_kv_heads=1), BF16, 9, 8, 3, fold, 80)           # 16 query heads per kv head
    if not fold:
        layer_case(slim, inputs.scaled(llama, dtype="fp32"), F32, 12, 9, 5, fold, 90)


def test_layer_is_replayed_from_a_graph(slim):
    wl = inputs.scaled(inputs.WORKLOADS["cfg2"], seq=1000, hidden=512, n_q_heads=8, n_kv_heads=2, ffn=1024)
    Hq, Hkv, d, block, n = wl.n_q_heads, wl.n_kv_heads, wl.head_dim, wl.block, wl.seq
    w = {k: v.cuda() for k, v in inputs.layer_weights(wl).items() if k not in ("g_attn", "g_ffn")}
    k, v = rand((n, Hkv, d), BF16, 1), rand((n, Hkv, d), BF16, 2)
    order = np.array([3, -1, 0, 15, 7], np.int32)
    pool, bos = pool_of(slim, k, v, block, 5, order, 3), torch.from_numpy(order).cuda()
    kr, vr = rand((4, Hkv, d), BF16, 4).cuda(), rand((4, Hkv, d), BF16, 5).cuda()
    shape = slim.make_shape(wl.hidden, Hq, Hkv, d, wl.ffn, block, wl.unit, wl.window, BF16, wl.rope_theta, wl.rms_eps)
    ws = torch.empty(slim.load_library().slim_decode_layer_workspace_bytes(ctypes.byref(shape), 5, 3), dtype=torch.uint8, device="cuda")
    x = rand((wl.hidden,), BF16, 6).cuda()
    call = lambda: slim.slim_decode_layer_kv4(shape, w, x, n + 3, pool, bos, n, kr, vr, 3, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z, q = call()
    for seed in range(3):
        x.copy_(rand((wl.hidden,), BF16, 10 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = z.clone(), q.clone()
        want = call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_from_prefill_to_a_follow_up_prompt(slim):
    """Every block is written in 4 bits, the active ones into slots and the others into the CPU pool; a decoding step scores, selects, swaps and attends; then the active blocks are read
    back in front of the answer's rows, and a follow-up prompt attends to all of it through a window with the first block in sight."""
    n, block, unit, Hq, Hkv, d, n_slots, n_keep = 2048 + 40, 64, 8, 32, 8, 128, 12, 10
    nb = -(-n // block)
    k, v = keys(n, Hkv, d, BF16, 11), rand((n, Hkv, d), BF16, 12)
    size = slim.kv4_block_bytes(block, Hkv, d)
    active = [0, 3, 4, 9, 10, 17, 20, 25, 30, nb - 1]
    sob, bos = np.full(nb, -1, np.int32), np.full(n_slots, -1, np.int32)
    for s, b in zip(np.random.default_rng(1).permutation(n_slots), active):
        sob[b], bos[s] = s, b
    slot_of_block, block_of_slot = torch.from_numpy(sob).cuda(), torch.from_numpy(bos).cuda()
    gpu_pool = torch.zeros(n_slots, size, dtype=torch.uint8, device="cuda")
    host_pool = torch.zeros(nb, size, dtype=torch.uint8).pin_memory()
    kd, vd = k.cuda(), v.cuda()
    for a, b in ((0, 1500), (1500, n)):                  # as a chunked prefill leaves them
        slim.slim_kv4_write(kd[a:b], vd[a:b], gpu_pool, block, slot_of_block, first_token=a)
        slim.slim_kv4_write(kd[a:b], vd[a:b], host_pool, block, first_token=a)
    k_rep = slim.slim_unit_keys(kd, block, unit)
    in_memory = torch.ones(nb, dtype=torch.int32, device="cuda")
    resp = 5
    kr, vr, q = keys(resp, Hkv, d, BF16, 13), rand((resp, Hkv, d), BF16, 14), rand((resp, Hq, d), BF16, 15, 0.5)
    scores = slim.slim_score_blocks_from_unit_keys(q[-4:].cuda().contiguous(), k_rep, n, Hkv, block, unit)
    cand = slim.slim_select_topk_blocks(scores, n_keep)
    info = slim.slim_kv_swap(cand, 0.9, slot_of_block, block_of_slot, in_memory, gpu_pool, host_pool)
    out = slim.slim_decode_attn_kv4(q[-1].cuda(), gpu_pool, block_of_slot, block, n, Hkv, kr.cuda(), vr.cuda())
    kept = cand.cpu().numpy()
    info = info.cpu().numpy()
    assert info[5] == 0 and info[2] == 1 and info[4] == len(set(kept.tolist()) - set(active))
    now = slot_of_block.cpu().numpy()
    assert set(np.nonzero(now >= 0)[0].tolist()) == set(kept.tolist())
    rows = so.kept_token_index(kept.astype(np.int64), block, n)
    kc, vc = ref.cached(ref.to64(k))[rows], ref.cached(ref.to64(v))[rows]
    kk, vv = np.concatenate([kc, ref.to64(kr)]), np.concatenate([vc, ref.to64(vr)])
    want, mag, reach = ref.attention(ref.to64(q[-1:]), kk, vv, np.ones((1, len(kk)), bool), 1 / math.sqrt(d))
    ref.within(out, want[0], ref.attention_bound(want, mag, reach, len(kk), d, BF16, vv)[0])
    # the follow-up prompt: 70 tokens behind the retained ones and the answer
    m, past = 70, len(rows) + resp
    kf, vf, qf = keys(m, Hkv, d, BF16, 16), rand((m, Hkv, d), BF16, 17), rand((m, Hq, d), BF16, 18, 0.5)
    k_all, v_all = torch.empty(past + m, Hkv, d, dtype=BF16, device="cuda"), torch.empty(past + m, Hkv, d, dtype=BF16, device="cuda")
    slim.slim_kv4_read(gpu_pool, block, n, slot_of_block, cand, k_out=k_all, v_out=v_all)
    np.testing.assert_array_equal(ref.to64(k_all[:len(rows)]), kc)
    np.testing.assert_array_equal(ref.to64(v_all[:len(rows)]), vc)
    k_all[len(rows):past], v_all[len(rows):past], k_all[past:], v_all[past:] = kr.cuda(), vr.cuda(), kf.cuda(), vf.cuda()
    window, sinks = 300, block
    got = slim.slim_sliding_attn(qf.cuda(), k_all, v_all, window, sinks)
    kk, vv = np.concatenate([kk, ref.to64(kf)]), np.concatenate([vv, ref.to64(vf)])
    p, j = np.arange(past, past + m)[:, None], np.arange(past + m)[None]
    seen = (j <= p) & ((j > p - window) | (j < sinks))
    want, mag, reach = ref.attention(ref.to64(qf), kk, vv, seen, 1 / math.sqrt(d))
    ref.within(got, want, ref.attention_bound(want, mag, reach, int(seen.sum(1).max()), d, BF16, vv))


def test_two_calls_at_once_on_streams_of_their_own(slim):
    """Attention over the same slots from two streams, each with its own workspace, beside a read of the slots: what each gives alone."""
    n, block, Hq, Hkv, d = 8192, 64, 32, 8, 128
    k, v = keys(n, Hkv, d, BF16, 1).cuda(), rand((n, Hkv, d), BF16, 2).cuda()
    pool = torch.zeros(128, slim.kv4_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv4_write(k, v, pool, block)
    order = torch.arange(128, dtype=torch.int32, device="cuda")
    qs = [rand((Hq, d), BF16, s).cuda() for s in (3, 4)]
    alone = [slim.slim_decode_attn_kv4(q, pool, order, block, n, Hkv) for q in qs]
    rows = slim.slim_kv4_read(pool, block, n, n_kv_heads=Hkv, head_dim=d)
    slide = slim.slim_sliding_attn(qs[0][None], k, v, 1000, 4)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    for turn in range(3):
        got = []
        for s, q in zip(streams, qs):
            with torch.cuda.stream(s):
                got.append(slim.slim_decode_attn_kv4(q, pool, order, block, n, Hkv))
        with torch.cuda.stream(streams[2]):
            again = slim.slim_kv4_read(pool, block, n, n_kv_heads=Hkv, head_dim=d)
        with torch.cuda.stream(streams[3]):
            other = slim.slim_sliding_attn(qs[0][None], k, v, 1000, 4)
        torch.cuda.synchronize()
        assert torch.equal(got[0], alone[0]) and torch.equal(got[1], alone[1]) and torch.equal(again[0], rows[0]) and torch.equal(again[1], rows[1]) and torch.equal(other, slide)
