"""The calls on a batch as a program makes them: step after step on lengths that stay on the GPU, in captured graphs, on several streams, with blocks that are swapped out, and up to a
follow-up prompt over the rows that are read back."""
import math

import numpy as np
import pytest
import torch

from tests import batch_reference as ref
from tests.kv4_reference import to64, within
from tests.test_gpu_kv4 import keys, rand, same

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def i32(x):
    return torch.tensor(np.asarray(x), dtype=I32).cuda()


class Batch:
    """State of a batch on the GPU and what a plain implementation makes of it."""

    def __init__(self, slim, R, block, Hq, Hkv, d, dtype, wide, n_slots, n_rows, seed):
        self.slim, self.R, self.block, self.Hq, self.Hkv, self.d, self.dtype, self.n_rows = slim, R, block, Hq, Hkv, d, dtype, n_rows
        self.order = np.random.default_rng(seed).permutation(n_slots)
        self.free, self.n_slots = i32(self.order), n_slots
        self.table, self.lens, self.used = i32(np.full((R, wide), -1)), i32(np.zeros(R)), i32([0])
        self.pool = torch.randint(0, 256, (n_slots, slim.kv8_block_bytes(block, Hkv, d)), dtype=torch.uint8, device="cuda")
        self.want_pool = self.pool.cpu().numpy()
        self.want = (np.zeros(R, np.int64), np.full((R, wide), -1), 0)
        need = slim.batch_attn_kv8_workspace_bytes(n_rows, R, Hq, Hkv, d)
        self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        z = lambda n: torch.zeros(n, dtype=I32, device="cuda")
        self.outs = dict(lens_out=z(R), row_start=z(R + 1), row_pos=z(n_rows), row_slot=z(n_rows), info=z(4))
        self.new = z(R)
        self.qkv = torch.zeros(n_rows, Hq + 2 * Hkv, d, dtype=dtype, device="cuda")
        self.out = torch.zeros(n_rows, Hq, d, dtype=dtype, device="cuda")
        self.theta = 10000.0

    def step(self):
        """One step on what lies in self.new and self.qkv."""
        s, Hq, Hkv = self.slim, self.Hq, self.Hkv
        lens, start, pos, slot, info = s.slim_batch_map(self.lens, self.new, self.block, self.table, self.free, self.n_slots, self.n_rows, used=self.used, **self.outs)
        q, k = self.qkv[:, :Hq].contiguous(), self.qkv[:, Hq:Hq + Hkv].contiguous()
        s.slim_rope(q, pos, self.theta)
        s.slim_rope(k, pos, self.theta)
        s.slim_kv8_write(k, self.qkv[:, Hq + Hkv:], self.pool, self.block, slot)
        s.slim_batch_attn_kv8(q, start, lens, self.table, self.pool, self.block, Hkv, out=self.out, workspace=self.workspace)
        self.q, self.k = q, k
        self.lens.copy_(lens)
        self.used.copy_(info[3:4])

    def put(self, new, seed):
        n = self.n_rows
        self.new.copy_(i32(new))
        x = torch.cat((rand((n, self.Hq, self.d), self.dtype, seed, 0.5), keys(n, self.Hkv, self.d, self.dtype, seed + 1), rand((n, self.Hkv, self.d), self.dtype, seed + 2)), 1)
        self.qkv.copy_(x)

    def check(self, new, attention=True):
        """Against the plain implementation, from the rotated rows that the GPU has formed (which another test holds to 64 bits)."""
        lens, table, used = self.want
        lens, start, pos, slot, info, table = ref.batch_map(lens.tolist(), list(new), table, self.order, used, self.block, self.n_slots, self.n_rows)
        self.want = (lens, table, int(info[3]))
        rows = int(start[-1])
        for name, x in (("lens_out", lens), ("row_start", start), ("row_pos", pos), ("row_slot", slot), ("info", info)):
            np.testing.assert_array_equal(self.outs[name].cpu().numpy(), x, err_msg=name)
        np.testing.assert_array_equal(self.table.cpu().numpy(), table)
        self.want_pool = ref.write(self.want_pool, to64(self.k)[:rows], to64(self.qkv[:, self.Hq + self.Hkv:])[:rows], slot[:rows], self.block)
        got = self.pool.cpu().numpy()
        H = self.Hkv
        for s in set((slot[:rows][slot[:rows] >= 0] // self.block).tolist()):
            np.testing.assert_array_equal(got[s], self.want_pool[s])
        if attention and rows:
            want = ref.attention(to64(self.q), start, lens, table, self.want_pool, self.block, H)
            within(self.out[:rows], want[0][:rows], ref.attention_bound(want, self.dtype)[:rows])


@pytest.mark.parametrize("Hq,Hkv,d,dtype,block", [(8, 2, 128, BF16, 16), (6, 2, 64, F32, 24), (7, 1, 128, BF16, 64)])
def test_steps_of_a_batch(slim, Hq, Hkv, d, dtype, block):
    """Prompts of odd lengths, then drafts and single tokens, some requests resting; the padding's rows stay as they were."""
    R = 6
    b = Batch(slim, R, block, Hq, Hkv, d, dtype, 500 // block + 2, 6 * 500 // block + 20, 320, 3)
    g = np.random.default_rng(0)
    for step in range(7):
        new = [100, 1, 0, 37, 64, 17] if step == 0 else [0, 0, 140, 3, 1, 1] if step == 1 else g.integers(0, 4, R).tolist()
        b.put(new, 10 * step)
        b.out.fill_(7.0)
        b.step()
        b.check(new)
        assert (b.out[sum(new):] == 7).all()


def test_a_captured_step_is_replayed_on_other_lengths(slim):
    """Lengths, tables and the list of free slots stay on the GPU: one graph serves every step.  A second graph of another batch shares the workspace."""
    R, block, Hq, Hkv, d = 5, 16, 8, 2, 128
    one, two = (Batch(slim, R, block, Hq, Hkv, d, BF16, 20, 120, 96, seed) for seed in (1, 2))
    two.workspace = one.workspace
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    new = [17, 1, 0, 30, 3]
    for i, b in enumerate((one, two)):
        b.put(new, 5 + i)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            b.step()
            side.synchronize()
            b.check(new)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                b.step()
        graphs.append(graph)
    torch.cuda.synchronize()
    # what the capture ran over was not executed: both batches are where the first step left them
    for turn, new in enumerate(([1, 1, 1, 1, 1], [0, 20, 7, 0, 2], [1, 0, 1, 0, 1], [40, 1, 30, 1, 1])):
        for i, (b, graph) in enumerate(zip((one, two), graphs)):
            b.put(new, 100 * turn + i)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            b.check(new)


def test_two_streams_with_their_own_workspaces(slim):
    R, block, Hq, Hkv, d = 4, 32, 8, 2, 128
    batches = [Batch(slim, R, block, Hq, Hkv, d, BF16, 40, 100, 512, seed) for seed in (1, 2)]
    for b in batches:
        b.put([300, 1, 100, 9], 3)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    for _ in range(1):
        for b, s in zip(batches, streams):
            with torch.cuda.stream(s):
                b.step()
    torch.cuda.synchronize()
    for b in batches:
        b.check([300, 1, 100, 9])


def test_blocks_that_are_swapped_out_are_not_attended_to(slim):
    """slim_kv_swap moves a request's blocks of 8 bits between the pool and host memory; its map of slots is the request's row of the table."""
    block, Hq, Hkv, d, nb = 32, 8, 2, 128, 12
    n = nb * block - 5
    size = slim.kv8_block_bytes(block, Hkv, d)
    k, v = keys(n, Hkv, d, BF16, 1), rand((n, Hkv, d), BF16, 2)
    host = torch.zeros(nb, size, dtype=torch.uint8).pin_memory()
    slim.slim_kv8_write(k.cuda(), v.cuda(), host, block, i32(np.arange(n)))
    torch.cuda.synchronize()
    want_pool = ref.write(np.zeros((nb, size), np.uint8), to64(k), to64(v), np.arange(n), block)
    np.testing.assert_array_equal(host.numpy(), want_pool)
    slots = 7
    pool = torch.full((slots, size), 255, dtype=torch.uint8, device="cuda")
    slot_of_block, block_of_slot, in_memory = i32(np.full(nb, -1)), i32(np.full(slots, -1)), i32(np.ones(nb))
    q = rand((3, Hq, d), BF16, 4).cuda()
    active = set()
    for candidates in ([0, 3, 4, 11], [0, 1, 2, 5, 6, 9, 11], [0, 11]):
        if len(active & set(candidates)) < len(candidates):          # (an overlap of gamma = 1 changes nothing: the last list is there already, among others)
            active = set(candidates)
        info = slim.slim_kv_swap(i32(candidates), 1.0, slot_of_block, block_of_slot, in_memory, pool, host)
        assert int(info[5]) == 0
        out = slim.slim_batch_attn_kv8(q, i32([0, 3]), i32([n]), slot_of_block[None], pool, block, Hkv)
        table = np.where(np.isin(np.arange(nb), list(active)), np.arange(nb), -1)[None]
        want = ref.attention(to64(q), [0, 3], [n], table, want_pool, block, Hkv)
        within(out, want[0], ref.attention_bound(want, BF16))


def test_a_follow_up_prompt_over_rows_that_are_read_back(slim):
    """The cache's rows in front of a prompt's own, for the attention of dense rows: the same as the attention over the pool up to the prompt's own rows, which there are 8 bits too."""
    n, m, block, Hq, Hkv, d = 700, 90, 64, 8, 2, 128
    k, v, q = keys(n + m, Hkv, d, BF16, 1), rand((n + m, Hkv, d), BF16, 2), rand((m, Hq, d), BF16, 3, 0.5).cuda()
    nb = slim.n_blocks(n + m, block)
    slots = np.random.default_rng(0).permutation(nb + 3)[:nb]
    p = np.arange(n + m)
    pool = torch.zeros(nb + 3, slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(slots[p // block] * block + p % block))
    kr, vr = slim.slim_kv8_read(pool, block, n + m, i32(slots), n_kv_heads=Hkv, head_dim=d)
    dense = slim.slim_sliding_attn(q, kr, vr, n + m)
    paged = slim.slim_batch_attn_kv8(q, i32([0, m]), i32([n + m]), i32(slots)[None], pool, block, Hkv)
    want = ref.attention(to64(q), [0, m], [n + m], slots[None], pool.cpu().numpy(), block, Hkv)
    bound = ref.attention_bound(want, BF16)
    within(dense, want[0], bound)
    within(paged, want[0], bound)


def test_many_requests_and_outputs_beyond_4_gb(slim):
    """4096 requests of 128 tokens, all of them rows of the step: 4.3 GB of queries and of results, tables of one shared pool.  The last requests against 64 bits."""
    R, n, block, Hq, Hkv, d = 4096, 128, 64, 32, 2, 128
    g = torch.Generator(device="cuda").manual_seed(0)
    pool = torch.zeros(2 * R, slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    lens, new, table = i32(np.zeros(R)), i32(np.full(R, n)), i32(np.full((R, 2), -1))
    lens, start, pos, slot, info = slim.slim_batch_map(lens, new, block, table, i32(np.arange(2 * R)[::-1].copy()), 2 * R, R * n)
    assert info.tolist() == [R * n, 2 * R, 0, 2 * R]
    k, v = (torch.randn(R * n, Hkv, d, dtype=BF16, device="cuda", generator=g) for _ in range(2))
    slim.slim_kv8_write(k, v, pool, block, slot)
    q = torch.randn(R * n, Hq, d, dtype=BF16, device="cuda", generator=g)
    assert q.nbytes >= 1 << 32
    out = slim.slim_batch_attn_kv8(q, start, lens, table, pool, block, Hkv)
    for r in (0, 2047, R - 2, R - 1):
        rows = slice(r * n, (r + 1) * n)
        slots = table[r].cpu().numpy()
        few = pool[torch.from_numpy(slots).cuda().long()].cpu().numpy()
        want = ref.attention(to64(q[rows]), [0, n], [n], np.array([[0, 1]]), few, block, Hkv)
        within(out[rows], want[0], ref.attention_bound(want, BF16))


def test_rows_far_apart(slim):
    """Queries and results 256 MB from row to row."""
    n, block, Hq, Hkv, d, ld = 20, 16, 4, 2, 128, 1 << 27
    room = torch.empty((n - 1) * ld + 2 * Hq * d, dtype=BF16, device="cuda")
    q, out = (room.as_strided((n, Hq, d), (ld, d, 1), at) for at in (0, Hq * d))
    q.copy_(rand((n, Hq, d), BF16, 1))
    k, v = keys(50, Hkv, d, BF16, 2), rand((50, Hkv, d), BF16, 3)
    pool = torch.zeros(4, slim.kv8_block_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
    slim.slim_kv8_write(k.cuda(), v.cuda(), pool, block, i32(np.arange(50)))
    slim.slim_batch_attn_kv8(q, i32([0, n]), i32([50]), i32([[0, 1, 2, 3]]), pool, block, Hkv, out=out)
    want = ref.attention(to64(q), [0, n], [50], np.arange(4)[None], pool.cpu().numpy(), block, Hkv)
    within(out, want[0], ref.attention_bound(want, BF16))
