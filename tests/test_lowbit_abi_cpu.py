"""Layouts and refusals of the 8-bit products and the block-sparse attention: every
call here returns on the host, none reaches the GPU."""
import pytest

from paper_2510_01565_amd import dit

P = 1 << 20  # a made-up, well aligned address
BF, F32 = dit.DIT_BF16, dit.DIT_F32
BAD, UNS, WS = dit.DIT_ERR_INVALID_ARG, dit.DIT_ERR_UNSUPPORTED, dit.DIT_ERR_WORKSPACE


def _err(fn, *args):
    with pytest.raises(dit.DitError) as e:
        fn(*args)
    assert dit.lib().dit_last_error().decode() != ""
    return e.value.status


@pytest.mark.parametrize("rows,K,block,codes,scales", [
    (1, 1, 1, 128, 4), (3, 128, 1, 384, 12), (3, 129, 1, 768, 12), (5, 640, 1, 3200, 40), (0, 64, 1, 0, 0),
    (1, 1, 128, 128, 4), (128, 513, 128, 128 * 640, 8), (129, 128, 128, 129 * 128, 8),
    (1 << 20, 1 << 12, 1, 1 << 32, 1 << 25),
])
def test_fp8_layout(rows, K, block, codes, scales):
    assert dit.fp8_layout(rows, K, block) == (codes, scales)


def test_fp8_shapes_are_checked():
    assert _err(dit.fp8_layout, -1, 8, 1) == BAD
    assert _err(dit.fp8_layout, 1, 0, 1) == BAD
    assert _err(dit.fp8_layout, 1, 8, 64) == BAD
    assert _err(dit.fp8_layout, 1, (1 << 24) + 1, 1) == UNS


def test_quantize_refusals():
    ok = [4, 64, 1, BF, P, P, P, 0]

    def bad(i, v):
        a = list(ok)
        a[i] = v
        return _err(dit.dit_quantize_fp8, *a)
    assert bad(0, -1) == BAD and bad(1, 0) == BAD and bad(2, 2) == BAD and bad(3, 2) == BAD
    assert bad(4, 0) == BAD and bad(5, 0) == BAD and bad(6, 0) == BAD        # NULL
    assert bad(4, P + 1) == BAD and bad(5, P + 8) == BAD and bad(6, P + 2) == BAD  # alignment
    dit.dit_quantize_fp8(0, 64, 1, BF, 0, 0, 0, 0)  # no rows: nothing to do


def test_linear_fp8_refusals():
    ok = [4, 8, 64, P, P, P, P, P, BF, P, BF, 0]

    def bad(i, v):
        a = list(ok)
        a[i] = v
        return _err(dit.dit_linear_fp8, *a)
    assert bad(0, -1) == BAD and bad(1, 0) == BAD and bad(2, 0) == BAD
    assert bad(2, (1 << 24) + 1) == UNS
    for i in (3, 4, 5, 6, 9):
        assert bad(i, 0) == BAD
    assert bad(3, P + 8) == BAD and bad(5, P + 8) == BAD and bad(4, P + 2) == BAD and bad(6, P + 1) == BAD
    assert bad(7, P + 1) == BAD and bad(9, P + 1) == BAD
    assert bad(8, 2) == BAD and bad(10, -1) == BAD
    dit.dit_linear_fp8(0, 8, 64, 0, 0, 0, 0, 0, BF, 0, BF, 0)


def test_linear_fp8_refuses_sides_and_outputs_past_its_offsets():
    def err(M, N):
        return _err(dit.dit_linear_fp8, M, N, 64, P, P, P, P, P, BF, P, BF, 0)
    top = (1 << 31) - 1
    assert err(1, top) == UNS and err(top, 1) == UNS and err(1, (1 << 30) + 1) == UNS and err((1 << 30) + 1, 1) == UNS
    assert err(1 << 18, (1 << 18) + 1) == UNS and err(65537, 1 << 20) == UNS


def _batch(*lens):
    """Requests of the given joint lengths, one image token and the rest text."""
    return dit.Batch([1] * len(lens), [1] * len(lens), [x - 1 for x in lens])


def test_block_counts_and_workspaces():
    assert dit.attention_query_blocks(_batch(1)) == 1
    assert dit.attention_query_blocks(_batch(128, 129, 1)) == 4
    # means of 3 + 1 query blocks and 5 + 1 key blocks (up to 16) in 64 bits
    assert dit.attention_select_workspace_size(_batch(300, 64), 3, 64, BF) == 4 * 3 * 64 * 8 + 16 * 3 * 64 * 8
    assert dit.attention_sparse_workspace_size(_batch(300, 64), 3, 64, BF) == 0
    most = dit.DIT_SPARSE_MAX_KEY_BLOCKS * dit.DIT_SPARSE_KEYS
    dit.attention_select_workspace_size(_batch(most), 1, 64, BF)
    assert _err(dit.attention_select_workspace_size, _batch(most + 1), 1, 64, BF) == UNS
    assert _err(dit.attention_sparse_workspace_size, _batch(5, most + 1), 1, 64, BF) == UNS
    assert _err(dit.attention_query_blocks, dit.Batch([0], [1], [1])) == BAD


def test_select_refusals():
    b = _batch(300, 64)
    n = dit.attention_select_workspace_size(b, 3, 64, BF)
    ok = [b, 3, 64, BF, P, P, 4, 0, P, P, n, 0]

    def bad(i, v):
        a = list(ok)
        a[i] = v
        return _err(dit.dit_attention_select, *a)
    assert bad(0, _batch()) == BAD
    assert bad(1, 0) == BAD and bad(1, 65536) == UNS and bad(2, 96) == UNS and bad(3, 5) == BAD
    assert _err(dit.dit_attention_select, b, 3, 128, F32, P, P, 4, 0, P, P, 1 << 30, 0) == UNS
    assert bad(6, 0) == BAD and bad(6, dit.DIT_SPARSE_MAX_KEY_BLOCKS + 1) == BAD and bad(7, 2) == BAD
    for i in (4, 5, 8):
        assert bad(i, 0) == BAD
    assert bad(4, P + 8) == BAD and bad(5, P + 8) == BAD and bad(8, P + 2) == BAD
    assert bad(9, 0) == WS and bad(9, P + 64) == WS and bad(10, n - 1) == WS


def test_sparse_refusals():
    b = _batch(300, 64)
    ok = [b, 3, 64, BF, P, P, P, P, 4, P, 0, 0, 0]

    def bad(i, v):
        a = list(ok)
        a[i] = v
        return _err(dit.dit_attention_sparse, *a)
    assert bad(0, _batch()) == BAD
    assert bad(1, -1) == BAD and bad(1, 65536) == UNS and bad(2, 32) == UNS and bad(3, 2) == BAD
    assert _err(dit.dit_attention_sparse, b, 3, 128, F32, P, P, P, P, 4, P, 0, 0, 0) == UNS
    assert bad(8, 0) == BAD and bad(8, -3) == BAD and bad(8, dit.DIT_SPARSE_MAX_KEY_BLOCKS + 1) == BAD
    for i in (4, 5, 6, 7, 9):
        assert bad(i, 0) == BAD
    for i in (4, 5, 6, 9):
        assert bad(i, P + 8) == BAD
    assert bad(7, P + 2) == BAD
    most = dit.DIT_SPARSE_MAX_KEY_BLOCKS * dit.DIT_SPARSE_KEYS
    assert bad(0, _batch(most + 1)) == UNS
