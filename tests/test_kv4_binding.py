"""What the binding of the calls on a cache in 4 bits refuses before it looks for a GPU (no GPU: the tensors lie on the host, and every refusal is named)."""
import pytest
import torch

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def slim():
    import os

    import paper_2508_06447_amd as slim
    if not os.path.exists(slim.LIB_PATH):
        from paper_2508_06447_amd.build import build_lib
        build_lib(verbose=False)
    return slim


def layer(slim, slots=3, in_pool=3, Hq=4, Hkv=2, hidden=256, rows=9, n_response=3, x=None, kr=None, dtype=BF16):
    """The arguments of slim_decode_layer_kv4 (the weights are looked at last)."""
    shape = slim.make_shape(hidden, Hq, Hkv, 128, 512, 16, 4, 8, dtype)
    pool = torch.zeros(in_pool, slim.kv4_block_bytes(16, Hkv, 128), dtype=torch.uint8)
    kr = torch.zeros(rows, Hkv, 128, dtype=dtype) if kr is None else kr
    return shape, {}, torch.zeros(hidden, dtype=dtype) if x is None else x, 60, pool, torch.full((slots,), -1, dtype=torch.int32), 48, kr, torch.zeros_like(kr), n_response


def test_a_map_of_more_slots_than_the_pool_has_is_refused(slim):
    """Every entry of the map that is not negative is an address in the pool."""
    q = torch.zeros(4, 128, dtype=BF16)
    for in_pool, slots in ((3, 4), (1, 2), (0, 1), (2, 1000)):
        pool = torch.zeros(in_pool, slim.kv4_block_bytes(16, 2, 128), dtype=torch.uint8)
        with pytest.raises(ValueError, match="slots"):
            slim.slim_decode_attn_kv4(q, pool, torch.zeros(slots, dtype=torch.int32), 16, 16 * slots, 2)
        with pytest.raises(ValueError, match="slots"):
            slim.slim_decode_layer_kv4(*layer(slim, slots=slots, in_pool=in_pool))
    # as many, and fewer: refused only for where they lie
    for slots in (3, 2):
        pool = torch.zeros(3, slim.kv4_block_bytes(16, 2, 128), dtype=torch.uint8)
        with pytest.raises(ValueError, match="GPU"):
            slim.slim_decode_attn_kv4(q, pool, torch.zeros(slots, dtype=torch.int32), 16, 16 * slots, 2)
        with pytest.raises(ValueError, match="GPU"):
            slim.slim_decode_layer_kv4(*layer(slim, slots=slots))


def test_response_rows_and_a_token_that_are_not_the_layers_are_refused(slim):
    """The layer writes row n_response and reads the others as [n_kv_heads, head_dim], and x_new as `hidden` channels of its own type."""
    for kr in (torch.zeros(9, 1, 128, dtype=BF16), torch.zeros(9, 2, 64, dtype=BF16), torch.zeros(9, 256, dtype=BF16), torch.zeros(9, 4, 128, dtype=BF16)):
        with pytest.raises(ValueError, match="response"):
            slim.slim_decode_layer_kv4(*layer(slim, kr=kr))
    with pytest.raises(ValueError, match="response"):
        slim.slim_decode_layer_kv4(*layer(slim, rows=3))                       # no row left for the token
    for x in (torch.zeros(255, dtype=BF16), torch.zeros(0, dtype=BF16), torch.zeros(2, 256, dtype=BF16)):
        with pytest.raises(ValueError, match="x_new"):
            slim.slim_decode_layer_kv4(*layer(slim, x=x))
    with pytest.raises(ValueError, match="x_new"):                              # tensors of one type, a layer of another
        slim.slim_decode_layer_kv4(*layer(slim, x=torch.zeros(256, dtype=BF16), kr=torch.zeros(9, 2, 128, dtype=BF16), dtype=F32))
    for x in (torch.zeros(256, dtype=BF16), torch.zeros(1, 256, dtype=BF16)):
        with pytest.raises(ValueError, match="GPU"):
            slim.slim_decode_layer_kv4(*layer(slim, x=x, rows=4))


def test_rows_of_a_list_of_blocks(slim):
    """Only the prompt's last block can be short, and only a list that ends with it has its rows."""
    from paper_2508_06447_amd.binding import _kv4_rows
    for n, block in ((74, 64), (65, 64), (64, 64), (128, 64), (1, 16), (205, 32)):
        nb = -(-n // block)
        assert _kv4_rows(n, block, None) == n
        for some in ([0], [nb - 1], list(range(nb)), list(range(nb - 1)), list(range(1, nb))):
            if some:
                want = sum(min(block, n - b * block) for b in some)
                assert _kv4_rows(n, block, torch.tensor(some, dtype=torch.int32)) == want, (n, block, some)


def test_an_empty_list_of_blocks_is_refused(slim):
    """An empty tensor has no address, and without a list every block is read."""
    pool, rows = torch.zeros(3, slim.kv4_block_bytes(16, 2, 128), dtype=torch.uint8), torch.zeros(48, 2, 128, dtype=BF16)
    none = torch.zeros(0, dtype=torch.int32)
    for more in (dict(k_out=rows, v_out=rows), dict(n_kv_heads=2, head_dim=128), dict(n_kv_heads=2, head_dim=128, n_out=48)):
        with pytest.raises(ValueError, match="blocks"):
            slim.slim_kv4_read(pool, 16, 48, blocks=none, **more)


def test_without_slots_there_need_be_no_pool(slim):
    """A token that attends to response rows alone."""
    none, q, r = torch.zeros(0, dtype=torch.int32), torch.zeros(4, 128, dtype=BF16), torch.zeros(5, 2, 128, dtype=BF16)
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        slim.slim_decode_attn_kv4(q, None, none, 16, 16, 2, r, r)
    args = list(layer(slim))
    args[4], args[5] = None, none
    with pytest.raises(ValueError, match="x_new must be a GPU tensor"):
        slim.slim_decode_layer_kv4(*args)


def test_rows_too_far_apart_for_the_entry_points_are_refused():
    """The distance of the rows is an int there: one of 2^32 elements and a row would be taken for a row."""
    from paper_2508_06447_amd.binding import _row_stride
    rows = lambda apart: torch.empty_strided((2, 8, 128), (apart, 128, 1), dtype=BF16, device="meta")
    assert _row_stride(rows(2**31 - 8), "k") == 2**31 - 8
    for apart in (2**31, 2**32 + 1024, 2**33 + 2048):
        with pytest.raises(ValueError, match="apart"):
            _row_stride(rows(apart), "k")
    assert _row_stride(rows(2**33)[:1], "k") == 1024                            # (one row is nowhere apart)
