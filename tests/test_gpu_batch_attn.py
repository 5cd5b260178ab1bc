"""Attention of a batch over its blocks in 8 bits, on the GPU, against a plain implementation in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import batch_reference as ref
from tests.kv4_reference import to64, within
from tests.test_gpu_kv4 import keys, rand

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def make(lens, new, block, Hkv, d, seed, at=0, kept=1.0, odd=True):
    """(pool, tables [R, blocks], row_start, lens with the rows) of requests; a fraction of the blocks is nowhere; bytes that are of no token are random, NaN among them."""
    g = np.random.default_rng(seed)
    total = [l + n for l, n in zip(lens, new)]
    nbs = [-(-t // block) for t in total]
    n_slots = sum(nbs) + 3
    size = ref.slot_bytes(block, Hkv, d)
    pool = g.integers(0, 256, (n_slots, at + size)).astype(np.uint8)
    if odd:
        pool[:, ::5] = 127
    order, used = g.permutation(n_slots), 0
    table = np.full((len(lens), max(nbs + [1]) + 2), 2**31 - 1)
    for r, t in enumerate(total):
        for b in range(nbs[r]):
            rows = min(block, t - b * block)
            x = keys(rows, Hkv, d, F32, seed + 31 * r + b).double().numpy(), rand((rows, Hkv, d), F32, seed + 31 * r + b + 7).double().numpy()
            slot = order[used]
            used += 1
            stale = pool[slot].copy()
            pool[slot:slot + 1] = ref.write(pool[slot:slot + 1], *x, np.arange(rows), block, at)
            for now, old in zip(ref.parts(pool[slot], block, Hkv, d, at)[:2], ref.parts(stale, block, Hkv, d, at)[:2]):
                now[:, rows:] = old[:, rows:]
            table[r, b] = slot if kept == 1.0 or g.random() < kept else (-1, n_slots, -5, 2**31 - 1)[int(g.integers(4))]
    start = np.concatenate([[0], np.cumsum(new)])
    return pool, table, start, np.array(total)


def run_case(slim, lens, new, block, Hq, Hkv, d, dtype, kept=1.0, pads=0, at=16, scale=0.0, q_scale=0.5, seed=None):
    seed = sum(lens) + block + Hq if seed is None else seed
    pool, table, start, total = make(lens, new, block, Hkv, d, seed, at, kept)
    n = int(start[-1]) + pads
    wide = rand((n, Hq + 2, d), dtype, seed + 1, q_scale).cuda()
    q = wide[:, 1:Hq + 1]
    out = torch.full((n, Hq + 1, d), 7.0, dtype=dtype, device="cuda")
    need = slim.batch_attn_kv8_workspace_bytes(n, len(lens), Hq, Hkv, d)
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    args = (i32(start), i32(total), i32(table), torch.from_numpy(pool).cuda(), block, Hkv)
    got = slim.slim_batch_attn_kv8(q, *args, softmax_scale=scale, layer_offset=at, out=out[:, :Hq], workspace=ws[:need])
    assert (ws[need:] == 255).all() and (out[:, Hq:] == 7).all() and (out[n - pads:] == 7).all()
    want = ref.attention(to64(q), start, total, table, pool, block, Hkv, at, scale or None)
    rows = int(start[-1])
    if rows:
        within(got[:rows], want[0][:rows], ref.attention_bound(want, dtype)[:rows])
    return q, args, got, want


CASES = [
    # tokens held, rows, block, Hq, Hkv, d, dtype
    ([0], [1], 16, 1, 1, 64, BF16),
    ([1], [1], 16, 4, 2, 128, F32),
    ([500], [1], 16, 4, 2, 64, F32),
    ([1000], [1], 64, 32, 8, 128, BF16),
    ([3000], [1], 64, 28, 4, 128, BF16),
    ([9000], [1], 128, 8, 1, 128, F32),
    ([70, 3, 0, 200, 64, 31, 32, 33], [1, 1, 1, 1, 1, 1, 1, 1], 32, 8, 2, 128, BF16),
    ([70, 3, 0, 200, 64], [0, 4, 1, 0, 1], 16, 6, 2, 64, BF16),
    (list(range(1, 71)), [1] * 70, 16, 4, 2, 64, BF16),
    ([40 * i % 700 for i in range(150)], [i % 4 for i in range(150)], 80, 4, 1, 64, F32),
    ([300], [5], 64, 32, 8, 128, BF16),
    ([300, 1000], [16, 3], 33, 14, 2, 128, BF16),
    ([0], [77], 7, 6, 2, 64, F32),
    ([0], [300], 64, 4, 2, 128, BF16),
    ([0, 129, 0], [200, 90, 65], 64, 7, 1, 128, BF16),
    ([777], [150], 80, 16, 1, 128, BF16),
    ([40], [129], 1, 2, 2, 64, BF16),
    ([333, 0], [100, 40], 300, 20, 2, 64, BF16),
    ([100], [70], 48, 17, 1, 128, F32),
    ([2000, 5, 64, 900], [1, 130, 1, 2], 64, 8, 2, 128, BF16),
    ([12000], [40], 64, 4, 1, 128, BF16),
    # more than 16 rows a request, and up to 64: tiles of 32 rows, some of them half empty
    ([5000], [13], 64, 8, 2, 128, BF16),
    ([600, 0, 31, 2000, 64, 1], [17, 16, 33, 32, 1, 15], 32, 4, 2, 64, BF16),
    ([90 * i % 1300 for i in range(90)], [1 + 7 * i % 12 for i in range(90)], 48, 10, 2, 128, BF16),
    ([40, 700, 0], [30, 100, 2], 16, 4, 2, 64, BF16),
    ([4000, 200], [3, 2], 64, 64, 8, 64, BF16),
    # more kv heads than workgroups run together: a share is all of a head's
    ([100, 3], [1, 4], 16, 160, 160, 64, BF16),
    ([50, 0], [90, 1], 16, 300, 300, 64, BF16),
    ([40], [12], 16, 1800, 900, 64, BF16),
    ([30], [2], 16, 800, 800, 64, F32),
    # a chunk of a prompt among requests of one token, in tiles of 256 rows and, too short for them, of 16
    ([37 * i % 400 for i in range(60)] + [500, 0], [1] * 60 + [140, 12], 64, 8, 2, 128, BF16),
    ([37 * i % 400 for i in range(60)] + [500, 0], [1] * 60 + [100, 12], 64, 8, 2, 128, BF16),
]


@pytest.mark.parametrize("lens,new,block,Hq,Hkv,d,dtype", CASES)
def test_attention(slim, lens, new, block, Hq, Hkv, d, dtype):
    print(f"batch attn lens={lens[:6]} new={new[:6]} block={block} {Hq}/{Hkv} d={d} {dtype}", flush=True)
    run_case(slim, lens, new, block, Hq, Hkv, d, dtype)


@pytest.mark.parametrize("lens,new,block,Hq,Hkv,d,dtype", CASES[3:])
def test_attention_over_retained_blocks(slim, lens, new, block, Hq, Hkv, d, dtype):
    print(f"batch attn, retained, lens={lens[:6]} new={new[:6]} block={block} {Hq}/{Hkv} d={d} {dtype}", flush=True)
    run_case(slim, lens, new, block, Hq, Hkv, d, dtype, kept=0.4, pads=3, scale=0.05)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_see_nothing_are_zero_and_padding_stays(slim, dtype):
    q, args, got, want = run_case(slim, [100, 0, 40], [3, 20, 30], 16, 8, 2, 128, dtype, kept=0.0, pads=5)
    assert (got[:53] == 0).all()
    # the first block is dropped: its own queries see nothing, later ones do
    pool, table, start, total = make([0], [64], 32, 2, 128, 3)
    table[0, 0] = -1
    q = rand((64, 8, 128), dtype, 4).cuda()
    out = slim.slim_batch_attn_kv8(q, i32(start), i32(total), i32(table), torch.from_numpy(pool).cuda(), 32, 2)
    assert (out[:32] == 0).all() and (out[32:].abs().amax(-1) > 0).all()
    # no request has rows
    out = slim.slim_batch_attn_kv8(q, i32([0, 0, 0]), i32([40, 0]), i32(np.zeros((2, 3))), torch.from_numpy(pool).cuda(), 32, 2)
    assert (out == 0).all()


@pytest.mark.parametrize("n,dtype", [(3, BF16), (14, BF16), (40, BF16), (200, BF16), (40, F32)])
def test_what_a_row_does_not_see_does_not_reach_it(slim, n, dtype):
    """Keys and values of later tokens that are not numbers, and exponents of blocks behind them."""
    lens, block, Hq, Hkv, d = 50, 16, 4, 2, 128
    pool, table, start, total = make([lens], [n], block, Hkv, d, 11, odd=False)
    q = rand((n, Hq, d), dtype, 5).cuda()
    args = lambda p, rows=n: (q[:rows], i32([0, rows]), i32([lens + rows]), i32(table), torch.from_numpy(p).cuda(), block, Hkv)
    clean = slim.slim_batch_attn_kv8(*args(pool))
    bad = pool.copy()
    for j in range(lens + 1, lens + n):                  # token j is seen by rows j - lens and later
        if j % 3 == 0:
            for x in ref.parts(bad[table[0, j // block]], block, Hkv, d)[:2]:
                x[:, j % block, j % d] = 127 if j % 2 else 255
    out = slim.slim_batch_attn_kv8(*args(bad))
    first = next(j for j in range(lens + 1, lens + n + 3) if j % 3 == 0) - lens
    # the same rows; the weights of one unit may have been added one by one instead of in a product
    want = ref.attention(to64(q), start, total, table, pool, block, Hkv)
    within(out[:first], want[0][:first], ref.attention_bound(want, dtype)[:first])
    assert torch.isfinite(out[:first]).all()
    assert torch.isnan(out[first:]).flatten(1).any(1).all() or first >= n
    assert torch.isfinite(clean).all()


@pytest.mark.parametrize("n,dtype", [(3, BF16), (14, BF16), (80, BF16), (14, F32)])
def test_a_query_that_is_not_a_number_is_its_own(slim, n, dtype):
    """One head of one query: the others of its tile are as they would be."""
    block, Hq, Hkv, d = 16, 4, 2, 128
    pool, table, start, total = make([50], [n], block, Hkv, d, 11, odd=False)
    q = rand((n, Hq, d), dtype, 5)
    q[1, 2, 7] = math.nan
    out = slim.slim_batch_attn_kv8(q.cuda(), i32(start), i32(total), i32(table), torch.from_numpy(pool).cuda(), block, Hkv)
    assert torch.isnan(out[1, 2]).all()
    q[1, 2] = 0.0
    out[1, 2] = 0.0
    want = ref.attention(to64(q), start, total, table, pool, block, Hkv)
    want[0][1, 2] = 0.0
    within(out, want[0], ref.attention_bound(want, dtype))


def test_large_and_flat_scores(slim):
    """Logits of some hundreds (one key takes everything) and equal keys (the mean of the values)."""
    n, block, Hkv, d = 640, 64, 2, 128
    v = rand((n, Hkv, d), F32, 2)
    k = torch.zeros(n, Hkv, d)
    k[:, :, 0] = 6.0
    k[400, :, :32] = 6.0
    q = torch.zeros(1, 8, d)
    q[0, 1, 0], q[0, 2, :32], q[0, 3, :32], q[0, 5] = 3.0, 18.0, -18.0, 100.0
    pool = torch.zeros(10, slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(np.arange(n)))
    for dtype in (F32, BF16):
        out = slim.slim_batch_attn_kv8(q.to(dtype).cuda(), i32([0, 1]), i32([n]), i32([np.arange(10)]), pool, block, Hkv)
        want = ref.attention(to64(q.to(dtype)), [0, 1], [n], np.arange(10)[None], pool.cpu().numpy(), block, Hkv)
        within(out, want[0], ref.attention_bound(want, dtype))


@pytest.mark.parametrize("n,dtype", [(1, BF16), (9, BF16), (40, BF16), (1, F32)])
def test_many_small_weights_beside_a_large_one(slim, n, dtype):
    """One key 12 to 21 binary places above 20000 others, whose values all have one sign: half of the sum to a hundredth of it, each weight beyond the places of a half-precision one."""
    block, Hq, Hkv, d, tokens = 64, 8, 2, 128, 20000
    v = rand((tokens, Hkv, d), F32, 2).abs() + 0.25
    k = torch.zeros(tokens, Hkv, d)
    k[77, :, 0] = 1.0
    q = torch.zeros(n, Hq, d)
    q[:, :, 0] = torch.linspace(12, 21, n * Hq).reshape(n, Hq) * math.log(2) * math.sqrt(d)
    nb = -(-tokens // block)
    pool = torch.zeros(nb, slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(np.arange(tokens)))
    q = q.to(dtype)
    out = slim.slim_batch_attn_kv8(q.cuda(), i32([0, n]), i32([tokens]), i32([np.arange(nb)]), pool, block, Hkv)
    want = ref.attention(to64(q), [0, n], [tokens], np.arange(nb)[None], pool.cpu().numpy(), block, Hkv)
    within(out, want[0], ref.attention_bound(want, dtype))


@pytest.mark.parametrize("n,dtype", [(1, BF16), (9, BF16), (40, BF16), (40, F32)])
def test_blocks_of_very_different_values(slim, n, dtype):
    """Blocks with Values of 0, 10^-12 to 10^12, in turn; queries that look at one kind of block, a token later at another."""
    block, Hq, Hkv, d, tokens = 16, 8, 2, 64, 900
    sizes = [0.0, 1.0, 1e-12, 1e12, 1e-6, 1e6]
    kind = np.arange(tokens) // block % len(sizes)
    v = rand((tokens, Hkv, d), F32, 2) * torch.tensor(sizes)[kind][:, None, None]
    k = rand((tokens, Hkv, d), F32, 3) * 0.1
    k[torch.arange(tokens), :, kind] += 8.0
    q = rand((n, Hq, d), F32, 4) * 0.1
    for i in range(n):
        for h in range(Hq):
            q[i, h, :len(sizes)] = 0.0
            q[i, h, (i + h) % len(sizes)] = 60.0         # 86 binary places above the others
    nb = -(-tokens // block)
    pool = torch.zeros(nb, slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(np.arange(tokens)))
    q = q.to(dtype)
    out = slim.slim_batch_attn_kv8(q.cuda(), i32([0, n]), i32([tokens]), i32([np.arange(nb)]), pool, block, Hkv)
    want = ref.attention(to64(q), [0, n], [tokens], np.arange(nb)[None], pool.cpu().numpy(), block, Hkv)
    for i in range(n):                                   # each row and head by the size of what it looks at
        for h in range(Hq):
            top = max(sizes[(i + h) % len(sizes)], 1e12 * 2.0 ** -80)
            part = (want[0][i:i + 1, h:h + 1], want[1][i:i + 1, h:h + 1], want[2], want[3], np.array([4.0 * top]))
            within(out[i:i + 1, h:h + 1], part[0], ref.attention_bound(part, dtype))


@pytest.mark.parametrize("new", [[1, 5, 70], [10, 5, 1]])
def test_results_do_not_depend_on_the_workspace_the_slots_or_the_call(slim, new):
    """The same bits again, from a workspace of other bytes and from slots in another order."""
    lens, block, Hq, Hkv, d = [900, 40, 3000], 64, 8, 2, 128
    pool, table, start, total = make(lens, new, block, Hkv, d, 1)
    n = sum(new)
    q = rand((n, Hq, d), BF16, 3).cuda()
    outs = []
    for seed in (0, 1, 2):
        g = np.random.default_rng(seed)
        order = g.permutation(pool.shape[0]) if seed else np.arange(pool.shape[0])
        moved = np.empty_like(pool)
        moved[order] = pool
        t = np.where((table >= 0) & (table < len(order)), order[np.clip(table, 0, len(order) - 1)], -1)
        ws = torch.full((slim.batch_attn_kv8_workspace_bytes(n, 3, Hq, Hkv, d),), 127 * seed, dtype=torch.uint8, device="cuda")
        outs.append(slim.slim_batch_attn_kv8(q, i32(start), i32(total), i32(t), torch.from_numpy(moved).cuda(), block, Hkv, workspace=ws))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]) and torch.isfinite(outs[0]).all()


@pytest.mark.parametrize("n_rows,dtype", [(1, BF16), (40, BF16), (300, BF16), (1, F32)])
def test_a_long_request_far_in_the_pool(slim, n_rows, dtype):
    """600000 tokens, slots behind 4 GB: what is seen by the last rows, from 64 bits on the GPU."""
    block, Hq, Hkv, d, n = 64, 8, 4, 128, 600_003
    size = slim.kv8_block_bytes(block, Hkv, d)
    nb = slim.n_blocks(n, block)
    n_slots = 2**32 // size + nb + 100
    g = torch.Generator(device="cuda").manual_seed(1)
    pool = torch.zeros(n_slots, size, dtype=torch.uint8, device="cuda")
    slots = torch.arange(n_slots - nb, n_slots, dtype=torch.int32, device="cuda")
    k, v = (torch.randn(n, Hkv, d, device="cuda", generator=g).to(BF16) for _ in range(2))
    p = torch.arange(n, device="cuda", dtype=torch.int64)
    slim.slim_kv8_write(k, v, pool, block, (slots.long()[p // block] * block + p % block).to(torch.int32))
    k, v = (x.double() for x in slim.slim_kv8_read(pool, block, n, slots, n_kv_heads=Hkv, head_dim=d))
    q = torch.randn(n_rows, Hq, d, device="cuda", generator=g).to(dtype)
    out = slim.slim_batch_attn_kv8(q, i32([0, n_rows]), i32([n]), slots[None], pool, block, Hkv)
    for i in {0, n_rows // 2, n_rows - 1}:
        last = n - n_rows + i + 1
        want, size_of, reach = torch.empty(Hq, d, dtype=torch.float64), torch.empty(Hq, d, dtype=torch.float64), 0.0
        for h in range(Hq):
            kk, vv = k[:last, h // 2], v[:last, h // 2]
            w = torch.softmax((kk @ q[i, h].double()) / math.sqrt(d), 0)
            want[h], size_of[h] = w @ vv, w @ vv.abs()
            reach = max(reach, float((kk.abs() @ q[i, h].double().abs()).max()) / math.sqrt(d))
        r = (want[None].numpy(), size_of[None].numpy(), reach, last, np.array([float(v.abs().max())]))
        within(out[i:i + 1], r[0], ref.attention_bound(r, dtype))


def test_binding_refusals(slim):
    pool, table, start, total = make([20, 5], [1, 2], 16, 2, 64, 1)
    q = rand((3, 4, 64), BF16, 1).cuda()
    good = dict(q=q, row_start=i32(start), lens=i32(total), block_table=i32(table), pool=torch.from_numpy(pool).cuda(), block=16, n_kv_heads=2)
    slim.slim_batch_attn_kv8(**good)
    for bad in (dict(row_start=i32(start[:-1])), dict(lens=i32(total[:1])), dict(block_table=i32(table[:1])), dict(block_table=i32(table.reshape(-1))), dict(lens=i32(total).cpu()),
                dict(out=q[:2]), dict(out=q.float()), dict(pool=torch.from_numpy(pool)), dict(q=q.cpu()), dict(q=q.transpose(0, 1)), dict(out=q.cpu()),
                dict(block_table=i32(table).t().contiguous().t())):
        with pytest.raises(ValueError):
            slim.slim_batch_attn_kv8(**{**good, **bad})
    for bad in (dict(row_start=i32(start).long()), dict(lens=i32(total).long()), dict(block_table=i32(table).long()), dict(q=q.half())):
        with pytest.raises(TypeError):
            slim.slim_batch_attn_kv8(**{**good, **bad})
    for bad in (dict(n_kv_heads=3), dict(n_kv_heads=0), dict(block=0), dict(block=17), dict(softmax_scale=-1.0), dict(softmax_scale=math.nan), dict(layer_offset=16), dict(layer_offset=8),
                dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(slim.SlimError):
            slim.slim_batch_attn_kv8(**{**good, **bad})
