"""A cache in 4 bits on the GPU: written, read back and attended to, against a plain implementation in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def rand(shape, dtype, seed, scale=1.0):
    g = np.random.default_rng(seed)
    return torch.from_numpy((scale * g.standard_normal(shape)).astype(np.float32)).to(dtype)


def keys(n, H, d, dtype, seed):
    """Rows whose channels and tokens differ in size, as keys' do."""
    g = np.random.default_rng(seed)
    x = g.standard_normal((n, H, d)) * np.exp2(g.integers(-2, 3, (n, 1, 1)))
    x[..., g.integers(0, d, 3)] *= 8
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def same(got: torch.Tensor, want: np.ndarray):
    """Equal values, NaN in the same places."""
    np.testing.assert_array_equal(ref.to64(got), want)


# ------------------------------------------------------------------------------------------- written and read back
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_rounding(slim, dtype):
    """Groups of every size of largest magnitude, filled with the values, the borders between them and their neighbours."""
    eps = torch.finfo(dtype).eps
    marks = np.concatenate([ref.GRID, (ref.GRID[1:] + ref.GRID[:-1]) / 2, [6.5, 6.99]])
    rows = []
    for e in list(range(-140, 128, 3)) + [-149, -127, -126, -125, -124, 124, 125, 126, 127]:
        for top in (1.0, 1.25, 1.5, 1.74, 1.75, 1.76, 1.99):
            m = np.concatenate([marks, marks * (1 + eps), marks * (1 - eps / 2)]) * np.exp2(min(max(e, -125), 125) - 2.0 if top < 1.75 else min(e + 1, 125) - 2.0)
            g = np.zeros(64)
            g[1:1 + 51][:len(m)] = np.minimum(m, top * 2.0 ** e)[:51] * np.where(np.arange(len(m[:51])) % 3 == 1, -1, 1)
            g[0], g[32] = top * 2.0 ** e, -top * 2.0 ** e
            rows.append(g)
    with np.errstate(over="ignore"):
        x = torch.from_numpy(np.array(rows)).to(F32).to(dtype)
    x = torch.where(torch.isfinite(x), x, torch.full_like(x, torch.finfo(dtype).max))
    k = x.view(-1, 1, 64).contiguous()
    v = k.flip(0).contiguous()
    pool = torch.zeros(-(-k.shape[0] // 16), slim.kv4_block_bytes(16, 1, 64), dtype=torch.uint8, device="cuda")
    slim.slim_kv4_write(k.cuda(), v.cuda(), pool, 16)
    kr, vr = slim.slim_kv4_read(pool, 16, k.shape[0], n_kv_heads=1, head_dim=64, dtype=dtype)
    want = ref.cached(ref.to64(k))
    bad = np.nonzero(ref.to64(kr) != want)
    assert not len(bad[0]), [(ref.to64(k)[i, h, c], ref.to64(kr)[i, h, c], want[i, h, c], np.abs(ref.to64(k)[i, h, c // 32 * 32:c // 32 * 32 + 32]).max()) for i, h, c in list(zip(*bad))[:8]]
    same(vr, ref.cached(ref.to64(v)))


@pytest.mark.parametrize("n,block,H,d,first,dtype", [
    (1, 16, 1, 32, 0, BF16), (1, 64, 8, 128, 9860, BF16), (17, 16, 2, 64, 5, F32), (200, 64, 8, 128, 0, BF16), (333, 80, 4, 128, 77, F32), (130, 1, 2, 64, 3, BF16),
    (129, 7, 3, 32, 11, F32), (1000, 128, 5, 128, 120, BF16), (65, 300, 2, 128, 250, BF16)])
def test_write_and_read_back(slim, n, block, H, d, first, dtype):
    print(f"kv4 write n={n} block={block} H={H} d={d} first={first} {dtype}", flush=True)
    nb = -(-(first + n) // block)
    g = np.random.default_rng(n)
    ns = nb + 3
    sob = g.permutation(ns)[:nb].astype(np.int32)
    size, at = ref.slot_bytes(block, H, d), 48
    k, v = keys(n, H, d, dtype, n), keys(n, H, d, dtype, n + 1)
    before = torch.from_numpy(g.integers(0, 256, (ns, at + size + 32)).astype(np.uint8))
    pool = before.cuda()
    out = slim.slim_kv4_write(k.cuda(), v.cuda(), pool, block, torch.from_numpy(sob).cuda(), first_token=first, layer_offset=at)
    assert out is pool
    # the bytes: those of the written rows as packed plainly, the others as they were
    pad = [np.zeros((first, H, d))]
    kk, vv = (np.concatenate(pad + [ref.to64(x)]) for x in (k, v))
    packed, want = ref.pack(kk, vv, block), before.numpy().copy()
    mark = ref.pack(np.concatenate([np.zeros((first, H, d)), np.ones((n, H, d))]), np.concatenate([np.zeros((first, H, d)), np.ones((n, H, d))]), block)
    touched = np.zeros_like(mark, dtype=bool)            # bytes of written rows: codes and exponents of ones are not zero, of zeros code 0 (and exponent byte 2)
    c, s = H * block * (d // 2), H * block * (d // 32)
    touched[:, :2 * c] = mark[:, :2 * c] != 0
    touched[:, 2 * c:2 * c + 2 * s] = mark[:, 2 * c:2 * c + 2 * s] > 2
    for b in range(nb):
        row = want[sob[b], at:at + size]
        row[touched[b]] = packed[b][touched[b]]
    got = pool.cpu().numpy()
    np.testing.assert_array_equal(got, want)
    # read back: the blocks that hold the chunk, as a list, into rows that are apart
    b0 = first // block
    rows = first + n - b0 * block
    wide = torch.full((rows + 2, H + 2, d), 7.0, dtype=dtype, device="cuda")
    kr, vr = slim.slim_kv4_read(pool, block, first + n, torch.from_numpy(sob).cuda(), torch.arange(b0, nb, dtype=torch.int32, device="cuda"),
                                k_out=wide[:rows, :H], v_out=torch.empty(rows, H, d, dtype=dtype, device="cuda"), layer_offset=at)
    part = first - b0 * block
    same(kr[part:], ref.cached(ref.to64(k)))
    same(vr[part:], ref.cached(ref.to64(v)))
    assert (wide[rows:] == 7).all() and (wide[:, H:] == 7).all()


def test_rows_of_a_fused_projection_are_written_as_they_lie(slim):
    n, Hq, H, d, block = 150, 4, 2, 128, 64
    qkv = keys(n, Hq + 2 * H, d, BF16, 3).cuda()
    k, v = qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    size = slim.kv4_block_bytes(block, H, d)
    a, b = (torch.zeros(3, size, dtype=torch.uint8, device="cuda") for _ in range(2))
    slim.slim_kv4_write(k, v, a, block)
    slim.slim_kv4_write(k.contiguous(), v.contiguous(), b, block)
    assert torch.equal(a, b) and a.any()


def test_a_prompt_written_in_chunks_and_token_by_token_is_the_same_cache(slim):
    n, H, d, block = 205, 4, 128, 32
    k, v = keys(n, H, d, BF16, 1).cuda(), keys(n, H, d, BF16, 2).cuda()
    size = slim.kv4_block_bytes(block, H, d)
    whole, parts = (torch.zeros(7, size, dtype=torch.uint8, device="cuda") for _ in range(2))
    sob = torch.tensor([3, 0, 6, 1, 5, 2, 4], dtype=torch.int32, device="cuda")
    slim.slim_kv4_write(k, v, whole, block, sob)
    cuts = [0, 1, 2, 33, 100, 101, 160, 204, 205]
    for a, b in zip(cuts, cuts[1:]):
        slim.slim_kv4_write(k[a:b], v[a:b], parts, block, sob, first_token=a)
    assert torch.equal(whole, parts)


def test_blocks_without_a_slot_are_left_out(slim):
    n, H, d, block = 100, 2, 64, 16
    k, v = keys(n, H, d, BF16, 1), keys(n, H, d, BF16, 2)
    sob = np.array([2, -1, 0, 99, 1, -7, 3], np.int32)
    pool = torch.full((4, slim.kv4_block_bytes(block, H, d)), 0x5a, dtype=torch.uint8, device="cuda")
    slim.slim_kv4_write(k.cuda(), v.cuda(), pool, block, torch.from_numpy(sob).cuda())
    packed = ref.pack(ref.to64(k), ref.to64(v), block)
    got = pool.cpu().numpy()
    for b in (0, 2, 4):
        np.testing.assert_array_equal(got[sob[b]], packed[b])
    ks, vs = torch.full((n, H, d), 7.0, dtype=BF16, device="cuda"), torch.full((n, H, d), 7.0, dtype=BF16, device="cuda")
    slim.slim_kv4_read(pool, block, n, torch.from_numpy(sob).cuda(), k_out=ks, v_out=vs)
    want = np.full((n, H, d), 7.0)
    for b in (0, 2, 4, 6):
        want[b * block:(b + 1) * block] = ref.cached(ref.to64(k))[b * block:(b + 1) * block]
    same(ks, want)
    # a list with entries outside the prompt, and an output with room for fewer rows
    lst = torch.tensor([-1, 0, 7, 4], dtype=torch.int32, device="cuda")
    ks.fill_(7.0)
    slim.slim_kv4_read(pool, block, n, torch.from_numpy(sob).cuda(), lst, k_out=ks[:59], v_out=vs[:59])
    want = np.full((n, H, d), 7.0)
    want[16:32] = ref.cached(ref.to64(k))[0:16]
    want[48:59] = ref.cached(ref.to64(k))[64:75]
    same(ks, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_groups_that_are_not_finite_read_back_as_nan(slim, dtype):
    k = keys(40, 2, 64, dtype, 4)
    k[3, 0, 5], k[7, 1, 40], k[11, 0, 63], k[12, 1, 0] = math.inf, -math.inf, math.nan, torch.finfo(dtype).max
    k[20] = 0.0
    k[21, :, 1:] = 0.0
    pool = torch.zeros(3, slim.kv4_block_bytes(16, 2, 64), dtype=torch.uint8, device="cuda")
    slim.slim_kv4_write(k.cuda(), k.cuda(), pool, 16)
    kr, vr = slim.slim_kv4_read(pool, 16, 40, n_kv_heads=2, head_dim=64, dtype=dtype)
    want = ref.cached(ref.to64(k))
    assert np.isnan(want).sum() == 3 * 32
    same(kr, want)
    same(vr, want)


def test_pinned_host_pool(slim):
    """Blocks that leave the GPU at once are written where the swap will look for them."""
    n, H, d, block = 100, 2, 128, 16
    k, v = keys(n, H, d, BF16, 5), keys(n, H, d, BF16, 6)
    host = torch.zeros(7, slim.kv4_block_bytes(block, H, d), dtype=torch.uint8).pin_memory()
    slim.slim_kv4_write(k.cuda(), v.cuda(), host, block)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(host.numpy(), ref.pack(ref.to64(k), ref.to64(v), block))
    kr, vr = slim.slim_kv4_read(host, block, n, n_kv_heads=H, head_dim=d)
    same(kr, ref.cached(ref.to64(k)))
    same(vr, ref.cached(ref.to64(v)))


def test_binding_refusals(slim):
    k = torch.zeros(16, 2, 64, dtype=BF16, device="cuda")
    pool = torch.zeros(1, slim.kv4_block_bytes(16, 2, 64), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        slim.slim_kv4_write(k, k[:8], pool, 16)
    with pytest.raises(ValueError):
        slim.slim_kv4_write(k.transpose(0, 1), k.transpose(0, 1), pool, 16)
    with pytest.raises(ValueError):
        slim.slim_kv4_write(k.cpu(), k.cpu(), pool, 16)
    with pytest.raises(TypeError):
        slim.slim_kv4_write(k, k, pool, 16, torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(TypeError):
        slim.slim_kv4_write(k.half(), k.half(), pool, 16)
    with pytest.raises(slim.SlimError):
        slim.slim_kv4_write(k, k, pool, 16, first_token=1)                       # behind the pool's only block
    with pytest.raises(ValueError):
        slim.slim_kv4_read(pool, 16, 17, torch.zeros(1, dtype=torch.int32, device="cuda"), n_kv_heads=2, head_dim=64)
    with pytest.raises(ValueError):
        slim.slim_kv4_read(pool, 16, 16, k_out=k[:8], v_out=k[:8])
    with pytest.raises(ValueError):
        slim.slim_kv4_read(pool, 16, 16, k_out=k)
    q, r = (torch.zeros(n, 2, 128, dtype=BF16, device="cuda") for n in (1, 5))
    pool = torch.zeros(1, slim.kv4_block_bytes(16, 2, 128), dtype=torch.uint8, device="cuda")
    slots = torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        slim.slim_decode_attn_kv4(q[0], pool, slots.long(), 16, 16, 2)
    with pytest.raises(ValueError):
        slim.slim_decode_attn_kv4(q[0], pool, slots, 16, 16, 2, out=q[0, :1])
    for k_resp, v_resp in ((r, None), (r, r[:4]), (r.float(), r.float()), (r.view(10, 1, 128), r.view(10, 1, 128))):
        with pytest.raises(ValueError):
            slim.slim_decode_attn_kv4(q[0], pool, slots, 16, 16, 2, k_resp, v_resp)
    shape, x = slim.make_shape(256, 2, 2, 128, 512, 16, 8, 16, BF16), torch.zeros(256, dtype=BF16, device="cuda")
    for k_resp, v_resp, n_resp in ((r, r[:4], 2), (r.float(), r.float(), 2), (r, r, 5)):
        with pytest.raises(ValueError):
            slim.slim_decode_layer_kv4(shape, {}, x, 20, pool, slots, 16, k_resp, v_resp, n_resp)


# ---------------------------------------------------------------------------------------------------- attention
def pool_of(slim, k, v, block, n_slots, order, seed, at=0):
    """Slots with the blocks `order` (slot -> block or -1) of the prompt; everything else random bytes, the NaN marker among them."""
    g = np.random.default_rng(seed)
    size = ref.slot_bytes(block, k.shape[1], k.shape[2])
    pool = g.integers(0, 256, (n_slots, at + size)).astype(np.uint8)
    pool[:, ::7] = 255
    packed = ref.pack(ref.to64(k), ref.to64(v), block)
    n = k.shape[0]
    H, d = k.shape[1:]
    for s, b in enumerate(order):
        if b >= 0:
            rows = min(block, n - b * block)
            part = packed[b].copy()
            keep = pool[s, at:at + size].copy()
            c, sc = H * block * (d // 2), H * block * (d // 32)
            for lo, width in ((0, d // 2), (c, d // 2), (2 * c, d // 32), (2 * c + sc, d // 32)):      # rows behind a short block's last one stay random
                a, z = part[lo:lo + H * block * width].reshape(H, block, width), keep[lo:lo + H * block * width].reshape(H, block, width)
                a[:, rows:] = z[:, rows:]
            pool[s, at:at + size] = part
    return torch.from_numpy(pool).cuda()


ATTN = [
    # prompt tokens, block, Hq, Hkv, slots, used, response, dtype
    (1, 16, 1, 1, 1, 1, 0, BF16),
    (64, 64, 4, 1, 1, 1, 0, F32),
    (1000, 64, 32, 8, 20, 16, 3, BF16),
    (1000, 64, 28, 4, 20, 13, 33, F32),
    (500, 80, 16, 1, 7, 6, 1, BF16),              # 16 query heads per kv head, blocks that end inside a unit
    (333, 7, 6, 2, 48, 48, 0, BF16),
    (77, 1, 2, 2, 77, 50, 2, F32),
    (5000, 128, 8, 8, 40, 39, 40, BF16),
    (3000, 33, 10, 2, 90, 80, 100, BF16),
    (16384, 64, 4, 1, 256, 250, 65, F32),
]


@pytest.mark.parametrize("n,block,Hq,Hkv,n_slots,used,resp,dtype", ATTN)
def test_decode_attention(slim, n, block, Hq, Hkv, n_slots, used, resp, dtype):
    print(f"kv4 decode n={n} block={block} {Hq}/{Hkv} slots={n_slots} used={used} resp={resp} {dtype}", flush=True)
    d, seed = 128, n + block
    g = np.random.default_rng(seed)
    k, v = keys(n, Hkv, d, dtype, seed), rand((n, Hkv, d), dtype, seed + 1)
    kr, vr = keys(resp, Hkv, d, dtype, seed + 2), rand((resp, Hkv, d), dtype, seed + 3)
    q = rand((Hq, d), dtype, seed + 4, 0.6)
    nb = -(-n // block)
    used = min(used, nb, n_slots)
    order = np.full(n_slots, -1, np.int32)
    blocks = np.concatenate([g.permutation(nb - 1)[:used - 1], [nb - 1]])
    order[g.permutation(n_slots)[:used]] = blocks
    stale = np.nonzero(order < 0)[0]
    bos = order.copy()
    if len(stale) > 1:
        bos[stale[0]] = nb + 5                           # a block that the prompt does not have
    pool = pool_of(slim, k, v, block, n_slots, order, seed, at=16)
    out = slim.slim_decode_attn_kv4(q.cuda(), pool, torch.from_numpy(bos).cuda(), block, n, Hkv, kr.cuda() if resp else None, vr.cuda() if resp else None, layer_offset=16)
    rows = np.concatenate([np.arange(b * block, min(n, (b + 1) * block)) for b in sorted(blocks)])
    kk = np.concatenate([ref.cached(ref.to64(k))[rows], ref.to64(kr)])
    vv = np.concatenate([ref.cached(ref.to64(v))[rows], ref.to64(vr)])
    want, size, reach = ref.attention(ref.to64(q)[None], kk, vv, np.ones((1, len(kk)), bool), 1 / math.sqrt(d))
    ref.within(out, want[0], ref.attention_bound(want, size, reach, len(kk), d, dtype, vv)[0])


def test_attention_does_not_depend_on_the_workspace_or_the_slots_order_of_free_bytes(slim):
    n, block, Hq, Hkv, d = 900, 64, 8, 2, 128
    k, v, q = keys(n, Hkv, d, BF16, 1), rand((n, Hkv, d), BF16, 2), rand((Hq, d), BF16, 3).cuda()
    order = np.array([-1, 4, 14, 3, -1, 0, 9], np.int32)
    outs = []
    for seed in (1, 2):
        pool = pool_of(slim, k, v, block, 7, order, seed)
        need = slim.load_library().slim_decode_attn_workspace_bytes(7, 0, Hq)
        ws = torch.full((need + 4096,), 255 * (seed - 1), dtype=torch.uint8, device="cuda")
        outs.append(slim.slim_decode_attn_kv4(q, pool, torch.from_numpy(order).cuda(), block, n, Hkv, workspace=ws[:need]))
        assert (ws[need:] == 255 * (seed - 1)).all()
    assert torch.equal(outs[0], outs[1]) and torch.isfinite(outs[0]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_token_that_sees_no_key_gets_zeros(slim, dtype):
    q = rand((8, 128), dtype, 1).cuda()
    size = slim.kv4_block_bytes(64, 2, 128)
    for ns in (3, 300):
        pool = torch.full((ns, size), 255, dtype=torch.uint8, device="cuda")
        out = slim.slim_decode_attn_kv4(q, pool, torch.full((ns,), -1, dtype=torch.int32, device="cuda"), 64, 500, 2, out=torch.full_like(q, 7.0))
        assert (out == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_group_that_is_not_finite_reaches_its_kv_heads_output(slim, dtype):
    n, block, Hq, Hkv, d = 200, 64, 4, 2, 128
    k, v, q = keys(n, Hkv, d, dtype, 1), rand((n, Hkv, d), dtype, 2), rand((Hq, d), dtype, 3).cuda()
    order = torch.arange(4, dtype=torch.int32).cuda()
    for x, bad_cols in ((k, slice(0, 128)), (v, slice(32, 64))):
        y = x.clone()
        y[150, 1, 40] = math.nan
        pool = torch.zeros(4, slim.kv4_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
        slim.slim_kv4_write((y if x is k else k).cuda(), (y if x is v else v).cuda(), pool, block)
        out = slim.slim_decode_attn_kv4(q, pool, order, block, n, Hkv).float()
        bad = torch.zeros(Hq, d, dtype=torch.bool)
        bad[2:, bad_cols] = True
        assert torch.equal(torch.isnan(out).cpu(), bad)


def test_large_and_flat_scores(slim):
    """Logits of +-300 (one key takes everything) and equal keys (the mean of the values)."""
    n, block, H, d = 640, 64, 2, 128
    v = rand((n, H, d), F32, 2)
    k = torch.zeros(n, H, d)
    k[:, :, 0] = 6.0
    k[400, :, :32] = 6.0
    q = torch.zeros(4, d)
    q[1, 0], q[2, :32], q[3, :32] = 3.0, 18.0, -18.0
    pool = torch.zeros(10, slim.kv4_block_bytes(block, H, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv4_write(k.cuda(), v.cuda(), pool, block)
    out = slim.slim_decode_attn_kv4(q.cuda(), pool, torch.arange(10, dtype=torch.int32).cuda(), block, n, H)
    kk, vv = ref.cached(ref.to64(k)), ref.cached(ref.to64(v))
    want, size, reach = ref.attention(ref.to64(q)[None], kk, vv, np.ones((1, n), bool), 1 / math.sqrt(d))
    ref.within(out, want[0], ref.attention_bound(want, size, reach, n, d, F32, vv)[0])


def test_attention_is_replayed_from_a_graph_on_a_stream_of_its_own(slim):
    n, block, Hq, Hkv, d = 4096, 64, 32, 8, 128
    k, v = keys(n, Hkv, d, BF16, 1).cuda(), rand((n, Hkv, d), BF16, 2).cuda()
    pool = torch.zeros(64, slim.kv4_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    order = torch.arange(64, dtype=torch.int32, device="cuda")
    q, out = rand((Hq, d), BF16, 3).cuda(), torch.zeros(Hq, d, dtype=BF16, device="cuda")
    kr, vr = keys(5, Hkv, d, BF16, 4).cuda(), rand((5, Hkv, d), BF16, 5).cuda()
    ws = torch.empty(slim.load_library().slim_decode_attn_workspace_bytes(64, 5, Hq), dtype=torch.uint8, device="cuda")
    ko, vo = torch.empty_like(k), torch.empty_like(v)

    def step():
        slim.slim_kv4_write(k, v, pool, block)
        slim.slim_decode_attn_kv4(q, pool, order, block, n, Hkv, kr, vr, out=out, workspace=ws)
        slim.slim_kv4_read(pool, block, n, k_out=ko, v_out=vo)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    for seed in range(4):
        k.copy_(keys(n, Hkv, d, BF16, 10 + seed))
        q.copy_(rand((Hq, d), BF16, 20 + seed))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, ko, vo)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, ko, vo)))
