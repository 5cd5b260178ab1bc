"""Attention of a batch over blocks whose Values differ widely, on the GPU, against 64 bits: what a key's block holds beside it, and what a row does not see, must not cost the row its result."""
import math

import numpy as np
import pytest
import torch

from tests import batch_reference as ref
from tests.kv4_reference import to64, within
from tests.test_gpu_kv4 import rand

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def attend(slim, q, k, v, block, rows_see=None):
    """(result, 64-bit reference) of the last len(q) of the tokens k, v."""
    n, Hkv, d = k.shape
    nb = -(-n // block)
    pool = torch.zeros(nb, slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(np.arange(n)))
    out = slim.slim_batch_attn_kv8(q.cuda(), i32([0, len(q)]), i32([n]), i32([np.arange(nb)]), pool, block, Hkv)
    return out, ref.attention(to64(q), [0, len(q)], [n], np.arange(nb)[None], pool.cpu().numpy(), block, Hkv)


# Rows of a kv head: 4 a query; above 64 they go in tiles of 256.
MANY = [(40, 64, BF16), (40, 128, BF16), (140, 128, BF16), (9, 128, BF16), (40, 64, F32)]


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("power", [6, 12, 13, 16, 20, 23, 26, 29, 60, 110])
def test_a_token_of_little_weight_and_large_values(slim, n, d, dtype, power):
    """Flat scores and Values about 1, one token with Values of 2^power whose weight is 10^-15 (2^-80 for the largest): it adds little, and its block's exponent must not push the others out."""
    tokens, block, Hq, Hkv = 640, 64, 8, 2
    v = rand((tokens, Hkv, d), F32, power) * 0.2 + 1.0
    v[5] = 2.0 ** power
    k = torch.zeros(tokens, Hkv, d)
    k[5, :, 0] = -1.0
    q = torch.zeros(n, Hq, d)
    q[:, :, 0] = (math.log(1e15) if power < 40 else 140 * math.log(2)) * math.sqrt(d)
    q = q.to(dtype)
    out, want = attend(slim, q, k, v, block)
    within(out, want[0], ref.attention_bound(want, dtype))


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("power", [13, 29, 100])
def test_a_later_token_with_large_values(slim, n, d, dtype, power):
    """A token that only the last rows see raises its block's exponent: the rows in front of it do not see it, and have the mean of the others."""
    held, block, Hq, Hkv = 700, 64, 8, 2
    tokens = held + n
    v = rand((tokens, Hkv, d), F32, 1) * 0.2 + 1.0
    later = tokens - 3
    v[later] = 2.0 ** power
    k = rand((tokens, Hkv, d), F32, 2) * 0.1
    q = rand((n, Hq, d), F32, 3).to(dtype)
    out, want = attend(slim, q, k, v, block)
    within(out, want[0], ref.attention_bound(want, dtype))
    assert (out[:n - 3].float() < 1.5).all()


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("tokens", [512, 3000])
@pytest.mark.parametrize("sizes", [[0.0, 1e20], [0.0, 1.0, 1e20, 1e30], [1e-30, 1e30], [0.0, 1.0]])
def test_blocks_of_zeros_count_in_the_sum(slim, n, d, dtype, tokens, sizes):
    """Equal scores, blocks with Values of 0 to 10^30 in turn: each key counts once, whatever its block's exponent."""
    block, Hq, Hkv = 16, 8, 2
    v = (rand((tokens, Hkv, d), F32, 2) * 0.2 + 1.0) * torch.tensor(sizes)[torch.arange(tokens) // block % len(sizes)][:, None, None]
    q = rand((n, Hq, d), F32, 3).to(dtype)
    out, want = attend(slim, q, torch.zeros(tokens, Hkv, d), v, block)
    within(out, want[0], ref.attention_bound(want, dtype))


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("tokens", [900, 3000])
def test_rows_that_look_at_one_kind_of_block(slim, n, d, dtype, tokens):
    """Blocks with Values of 10^-30 to 10^30, and queries that look at one kind each, some 86 binary places above the others: results of every size beside each other."""
    block, Hq, Hkv = 16, 8, 2
    sizes = [1.0, 1e-30, 1e20, 1e-12, 1e30, 1e6]
    kind = np.arange(tokens) // block % len(sizes)
    v = rand((tokens, Hkv, d), F32, 2) * torch.tensor(sizes)[kind][:, None, None]
    k = rand((tokens, Hkv, d), F32, 3) * 0.1
    k[torch.arange(tokens), :, kind] += 8.0
    q = rand((n, Hq, d), F32, 4) * 0.1
    q[:, :, :len(sizes)] = 0.0
    for i in range(n):
        for h in range(Hq):
            q[i, h, (i + h) % len(sizes)] = 60.0 * math.sqrt(d / 64)
    q = q.to(dtype)
    out, want = attend(slim, q, k, v, block)
    bound = ref.attention_bound(want, dtype)
    rest = want[3] * 2.0 ** -126 * want[4].max()         # what weights below the smallest normal number leave out is of the largest Values' size
    assert rest < 1e-3
    within(out, want[0], bound)


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("apart", [False, True])
def test_values_that_are_not_numbers_are_seen_by_their_rows_alone(slim, n, d, dtype, apart):
    """A token with a Value that is not a number, at places all over a tile of keys and in channels of every lane: rows in front of it are as they would be, later ones are not numbers.
    Blocks alike, or too far apart for float16."""
    held, block, Hq, Hkv = 150, 16, 8, 2
    tokens = held + n
    nb = -(-tokens // block)
    v = rand((tokens, Hkv, d), F32, 2) * torch.tensor([1.0, 2.0 ** -20 if apart else 1.0])[torch.arange(tokens) // block % 2][:, None, None]
    k = rand((tokens, Hkv, d), F32, 3)
    q = rand((n, Hq, d), F32, 4).to(dtype)
    pool = torch.zeros(nb, slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(np.arange(tokens)))
    clean = pool.cpu().numpy()
    want = ref.attention(to64(q), [0, n], [tokens], np.arange(nb)[None], clean, block, Hkv)
    bound = ref.attention_bound(want, dtype)
    for j in list(range(held, tokens - 1, 7)) + [tokens - 1]:
        bad = clean.copy()
        ref.parts(bad[j // block], block, Hkv, d)[1][:, j % block, (5 * j) % d] = 127 if j % 2 else 255
        out = slim.slim_batch_attn_kv8(q.cuda(), i32([0, n]), i32([tokens]), i32([np.arange(nb)]), torch.from_numpy(bad).cuda(), block, Hkv)
        first = j - held                                 # row i is token held + i
        within(out[:first], want[0][:first], bound[:first]) if first else None
        assert torch.isnan(out[first:]).any(-1).all()
        assert torch.isfinite(out[:first]).all()


def test_calls_that_overlap_on_two_streams(slim):
    """Both streams' queues are filled behind a kernel that runs longer than that takes; every call's bits are those of the same calls one behind the other."""
    block, Hq, Hkv, d, steps = 32, 8, 2, 128, 6
    work = []
    for seed in (1, 2):
        lens, new = [600 * seed, 40, 2000], [180, 1, 30 * seed]
        total = [l + m for l, m in zip(lens, new)]
        nbs = [-(-t // block) for t in total]
        table = np.full((3, max(nbs)), -1)
        order, at = np.random.default_rng(seed).permutation(sum(nbs)), 0
        for r, nb in enumerate(nbs):
            table[r, :nb], at = order[at:at + nb], at + nb
        slots = np.concatenate([table[r][np.arange(l, t) // block] * block + np.arange(l, t) % block for r, (l, t) in enumerate(zip(lens, total))])
        pool = torch.zeros(sum(nbs), slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
        slim.slim_kv8_write(rand((sum(nbs) * block, Hkv, d), BF16, seed).cuda(), rand((sum(nbs) * block, Hkv, d), BF16, seed + 5).cuda(), pool, block, i32(np.arange(sum(nbs) * block)))
        n = sum(new)
        kvs = [(rand((n, Hkv, d), BF16, 10 * seed + s).cuda(), rand((n, Hkv, d), BF16, 20 * seed + s).cuda()) for s in range(steps)]
        qs = [rand((n, Hq, d), BF16, 30 * seed + s).cuda() for s in range(steps)]
        ws = torch.empty(slim.batch_attn_kv8_workspace_bytes(n, 3, Hq, Hkv, d), dtype=torch.uint8, device="cuda")
        args = (i32(np.concatenate([[0], np.cumsum(new)])), i32(total), i32(table))
        work.append((pool, i32(slots), kvs, qs, ws, args))

    def step(w, s, out):
        pool, slots, kvs, qs, ws, args = w
        slim.slim_kv8_write(*kvs[s], pool, block, slots)
        slim.slim_batch_attn_kv8(qs[s], *args, pool, block, Hkv, out=out, workspace=ws)

    start = [w[0].clone() for w in work]
    want = [[torch.zeros_like(w[3][s]) for s in range(steps)] for w in work]
    for w, outs in zip(work, want):
        for s in range(steps):
            step(w, s, outs[s])
    for w, pool in zip(work, start):
        w[0].copy_(pool)
    got = [[torch.zeros_like(w[3][s]) for s in range(steps)] for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for stream in streams:
        with torch.cuda.stream(stream):
            torch.cuda._sleep(20_000_000)                # 10 ms at least
    for s in range(steps):
        for w, outs, stream in zip(work, got, streams):
            with torch.cuda.stream(stream):
                step(w, s, outs[s])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for s in range(steps):
            assert torch.equal(a[s], b[s]) and torch.isfinite(a[s]).all()


@pytest.mark.parametrize("n,d,dtype", MANY)
@pytest.mark.parametrize("tokens", [640, 2500])
@pytest.mark.parametrize("at", [5, 333, 470])
@pytest.mark.parametrize("places", [20.4, 24.4, 28.4, 32.4, 40.4, 70.4])
def test_a_key_that_takes_nearly_everything_and_has_no_value(slim, n, d, dtype, tokens, places, at):
    """One key `places` binary places above the others, its Values zeros: the result is of the others alone, whose weights are far below a float16's beside it."""
    block, Hq, Hkv = 64, 8, 2
    v = rand((tokens, Hkv, d), F32, int(places)) * 0.2 + 1.0
    v[at] = 0.0
    k = torch.zeros(tokens, Hkv, d)
    k[at, :, 0] = 1.0
    q = torch.zeros(n, Hq, d)
    q[:, :, 0] = places * math.log(2) * math.sqrt(d)
    q = q.to(dtype)
    out, want = attend(slim, q, k, v, block)
    within(out, want[0], ref.attention_bound(want, dtype))
