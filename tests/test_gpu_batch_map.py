"""The tables of a batch's step on the GPU against a plain loop."""
import numpy as np
import pytest
import torch

from tests import batch_reference as ref

pytestmark = pytest.mark.gpu
I32 = torch.int32


@pytest.fixture(scope="module")
def slim():
    import paper_2508_06447_amd as slim
    slim.load_library()
    return slim


def i32(x):
    return torch.tensor(np.asarray(x), dtype=I32).cuda()


def check(slim, lens, new, block, wide, n_free, used, n_slots, n_rows, seed=0, table=None, free=None):
    g = np.random.default_rng(seed)
    R = len(lens)
    table = g.integers(-2, n_slots + 3, (R, wide)) if table is None else table
    free = g.permutation(max(n_slots, n_free))[:n_free] if free is None else free
    want = ref.batch_map(list(map(int, lens)), list(map(int, new)), table, free, used, block, n_slots, n_rows)
    t = i32(table)
    got = slim.slim_batch_map(i32(lens), i32(new), block, t, i32(free), n_slots, n_rows, used=i32([used]),
                              row_pos=torch.full((n_rows,), 77, dtype=I32, device="cuda"), row_slot=torch.full((n_rows,), 77, dtype=I32, device="cuda"))
    for name, a, b in zip(("lens_out", "row_start", "row_pos", "row_slot", "info", "table"), (*got, t), want):
        np.testing.assert_array_equal(a.cpu().numpy(), b, err_msg=name)
    return want


@pytest.mark.parametrize("R,block,longest,most,n_rows", [
    (1, 16, 0, 1, 1), (1, 64, 500, 1, 1), (1, 1, 7, 300, 512), (3, 7, 20, 40, 128), (64, 16, 300, 1, 64), (65, 64, 1000, 1, 80), (256, 64, 8192, 1, 256), (256, 16, 400, 30, 8192),
    (300, 33, 100, 5, 2000), (1000, 64, 2000, 2, 2048), (4096, 16, 64, 3, 20000), (5, 64, 100, 9000, 50000), (2, 128, 0, 200000, 400000)])
def test_steps(slim, R, block, longest, most, n_rows):
    print(f"map R={R} block={block} longest={longest} most={most} rows={n_rows}", flush=True)
    g = np.random.default_rng(R + block)
    lens, new = g.integers(0, longest + 1, R), g.integers(0, most + 1, R)
    lens[g.integers(0, R)] = longest // block * block                           # a block that is just full
    new[g.integers(0, R)] = most
    while new.sum() > n_rows:
        new //= 2
    wide = int(-(-(lens + new).max() // block)) + 2
    taken = int((-(-(lens + new) // block) - -(-lens // block)).sum())
    want = check(slim, lens, new, block, wide, taken + 7, 7, taken + 100, n_rows, seed=R)
    assert want[4].tolist() == [int(new.sum()), taken, 0, 7 + taken]


def test_requests_that_rest_and_a_batch_without_rows(slim):
    check(slim, [0, 5, 16, 17, 0], [0, 0, 0, 0, 0], 16, 4, 3, 1, 20, 8)
    check(slim, [0, 5, 16, 17, 0], [0, 3, 0, 1, 0], 16, 4, 3, 1, 20, 8)
    check(slim, [0] * 70 + [5], [0] * 70 + [12], 16, 2, 1, 0, 20, 64)


def test_every_row_and_the_last_free_slot(slim):
    """Exactly as many rows and slots as there are."""
    check(slim, [16, 31, 0], [1, 2, 33], 16, 3, 5, 0, 9, 36)
    check(slim, [16, 31, 0], [1, 2, 33], 16, 3, 8, 3, 9, 36)
    check(slim, [0], [48], 16, 3, 3, 0, 9, 48)


@pytest.mark.parametrize("lens,new,wide,n_free,used,n_rows,bits", [
    ([3, -1, 4], [1, 1, 1], 2, 9, 0, 8, 1), ([3, 1, 4], [1, -1, 1], 2, 9, 0, 8, 1), ([3, 30, 4], [1, 3, 1], 2, 9, 0, 8, 1), ([3, 30, 4], [1, 2, 6], 2, 9, 0, 8, 2),
    ([16, 16, 0], [1, 1, 1], 2, 2, 0, 8, 4), ([16, 16, 0], [1, 1, 1], 2, 9, 7, 8, 4), ([16, 16, 0], [1, 1, 1], 2, 9, -1, 8, 4), ([0, 16, -5], [20, 1, 1], 2, 1, 0, 8, 7),
    ([2**31 - 1, 0], [2**31 - 1, 1], 2, 9, 0, 8, 1), ([0] * 3, [2**24 - 1] * 3, 1 << 20, 9, 0, 8, 6), ([0] * 3, [1, 2, 3], 2, 9, 2**31 - 1, 8, 4)])
def test_errors_leave_a_step_without_rows(slim, lens, new, wide, n_free, used, n_rows, bits):
    want = check(slim, lens, new, 16, wide, n_free, used, 20, n_rows, table=np.full((len(lens), wide), 3) if wide > 1000 else None)
    assert want[4].tolist() == [0, 0, bits, used] and (want[3] == -1).all()


def test_entries_outside_the_pool_have_no_place(slim):
    table = np.array([[-1, 5, 20, 7, 9, 9], [2**31 - 1, -2**31, 0, 19, 9, 9]])
    want = check(slim, [30, 0], [30, 64], 16, 6, 8, 0, 20, 128, table=table, free=np.array([-3, 4, 100, 2**31 - 1, 6, 1, 2, 3]))
    assert (want[3][:94] == -1).any() and (want[3][:94] >= 0).any()


def test_places_up_to_32_bits(slim):
    n_slots = (2**31 - 1) // 64
    check(slim, [0, 100], [130, 1], 64, 4, 4, 0, n_slots, 200, table=np.array([[9, 9, 9, 9], [0, n_slots - 1, 9, 9]]), free=np.array([n_slots - 1, n_slots - 2, n_slots, 0]))


def test_without_a_count_of_taken_slots_and_step_after_step(slim):
    """A hundred steps, each on what the one before has left; the lengths stay on the GPU."""
    R, block, wide = 37, 16, 40
    g = np.random.default_rng(0)
    free = g.permutation(900)
    lens, table, used = np.zeros(R, np.int64), np.full((R, wide), -1), 0
    at, t, f, u = i32(lens), i32(table), i32(free), None
    for step in range(100):
        new = g.integers(0, 300, R) // 100 if step else g.integers(0, 100, R)
        lens, start, pos, slot, info, table = ref.batch_map(lens.tolist(), new.tolist(), table, free, used, block, 900, 4096)
        used = int(info[3])
        at, *got = slim.slim_batch_map(at, i32(new), block, t, f, 900, 4096, used=u)
        u = got[3][3:4]
        if step % 9 == 0 or step == 99:
            for a, b in zip((at, *got, t), (lens, start, pos, slot, info, table)):
                np.testing.assert_array_equal(a.cpu().numpy(), b)
    held = table[table >= 0]
    assert len(set(held.tolist())) == len(held) == used


def test_binding_refusals(slim):
    z = lambda n: torch.zeros(n, dtype=I32, device="cuda")
    good = dict(lens=z(3), n_new=z(3), block=16, block_table=z(12).view(3, 4), free_slots=z(5), n_slots=20, n_rows=8)
    slim.slim_batch_map(**good)
    for bad in (dict(n_new=z(2)), dict(used=z(2)), dict(lens_out=z(4)), dict(row_start=z(3)), dict(row_pos=z(9)), dict(row_slot=z(7)), dict(info=z(3)), dict(lens=z(3).cpu()),
                dict(block_table=z(16).view(4, 4)[:3].t()[:3]), dict(block_table=z(24).view(3, 8)[:, ::2])):
        with pytest.raises(ValueError):
            slim.slim_batch_map(**{**good, **bad})
    for bad in (dict(lens=z(3).long()), dict(n_new=z(3).float()), dict(free_slots=z(5).long()), dict(used=z(1).long()), dict(row_slot=z(8).long())):
        with pytest.raises(TypeError):
            slim.slim_batch_map(**{**good, **bad})
    info = z(4)
    for bad in (dict(n_rows=0), dict(block=0), dict(info=info, used=info[3:4]), dict(lens_out=good["lens"]), dict(n_slots=0)):
        with pytest.raises(slim.SlimError):
            slim.slim_batch_map(**{**good, **bad})
