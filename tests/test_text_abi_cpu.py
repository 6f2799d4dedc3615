"""Layouts, frequencies and refusals of the 4-bit products, the rotary positions and the grouped attention: every call
here returns on the host, none reaches the GPU."""
import random

import pytest

from paper_2510_01565_amd import dit

P = 1 << 20  # a made-up, well aligned address
BF, F32 = dit.DIT_BF16, dit.DIT_F32
BAD, UNS, WS = dit.DIT_ERR_INVALID_ARG, dit.DIT_ERR_UNSUPPORTED, dit.DIT_ERR_WORKSPACE
INF, NAN = float("inf"), float("nan")


def _err(fn, *args):
    with pytest.raises(dit.DitError) as e:
        fn(*args)
    assert dit.lib().dit_last_error().decode() != ""
    return e.value.status


def _refusals(fn, ok):
    def bad(*changes):
        a = list(ok)
        for i, v in changes:
            a[i] = v
        return _err(fn, *a)
    return bad


@pytest.mark.parametrize("rows,K,codes,scales", [
    (1, 1, 128, 16), (3, 256, 384, 48), (3, 257, 768, 48), (5, 512, 1280, 80), (5, 513, 1920, 160), (0, 64, 0, 0),
    (1 << 21, 1 << 12, 1 << 32, 1 << 28),
])
def test_fp4_layout(rows, K, codes, scales):
    assert dit.fp4_layout(rows, K) == (codes, scales)


def test_fp4_shapes_are_checked():
    assert _err(dit.fp4_layout, -1, 8) == BAD
    assert _err(dit.fp4_layout, 1, 0) == BAD
    assert _err(dit.fp4_layout, 1, (1 << 22) + 1) == UNS
    assert _err(dit.fp4_layout, (1 << 18) + 1, 1 << 22) == UNS and dit.fp4_layout(1 << 18, 1 << 22) == (1 << 39, 1 << 35)


def test_quantize_fp4_refusals():
    bad = _refusals(dit.dit_quantize_fp4, [4, 64, BF, P, P, P, 0])
    assert bad((0, -1)) == BAD and bad((1, 0)) == BAD and bad((1, (1 << 22) + 1)) == UNS and bad((2, 2)) == BAD
    for i in (3, 4, 5):
        assert bad((i, 0)) == BAD
    assert bad((3, P + 1)) == BAD and bad((4, P + 8)) == BAD and bad((5, P + 4)) == BAD
    dit.dit_quantize_fp4(0, 64, BF, 0, 0, 0, 0)  # no rows: nothing to do


def test_dequantize_fp4_refusals():
    bad = _refusals(dit.dit_dequantize_fp4, [4, 64, P, P, F32, P, 0])
    assert bad((0, -1)) == BAD and bad((1, 0)) == BAD and bad((1, (1 << 22) + 1)) == UNS and bad((4, -1)) == BAD
    for i in (2, 3, 5):
        assert bad((i, 0)) == BAD
    assert bad((2, P + 8)) == BAD and bad((3, P + 4)) == BAD and bad((5, P + 2)) == BAD
    dit.dit_dequantize_fp4(0, 64, 0, 0, BF, 0, 0)


def test_linear_fp4_refusals():
    bad = _refusals(dit.dit_linear_fp4, [4, 8, 64, P, P, P, P, P, BF, P, BF, 0])
    assert bad((0, -1)) == BAD and bad((1, 0)) == BAD and bad((2, 0)) == BAD and bad((2, (1 << 22) + 1)) == UNS
    for i in (3, 4, 5, 6, 9):
        assert bad((i, 0)) == BAD
    for i in (3, 4, 5, 6):
        assert bad((i, P + 8)) == BAD
    assert bad((7, P + 1)) == BAD and bad((9, P + 1)) == BAD and bad((8, 2)) == BAD and bad((10, -1)) == BAD
    top = (1 << 31) - 1
    assert bad((0, 1), (1, top)) == UNS and bad((0, top), (1, 1)) == UNS and bad((0, 65537), (1, 1 << 20)) == UNS
    dit.dit_linear_fp4(0, 8, 64, 0, 0, 0, 0, 0, BF, 0, BF, 0)


def test_rope_frequencies():
    w = list(dit.rope_frequencies(8, 10000.0))
    assert w == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-14)
    # a hundred thousand positions: 15915, 1591, 159 and 15.9 turns
    w = list(dit.rope_frequencies(8, 10000.0, 4.0, 1e5, 100.0, 1000.0))
    g = (159.15494309189535 - 100) / 900
    assert w == pytest.approx([1.0, 0.1, 0.01 * (g + (1 - g) / 4), 0.001 / 4], rel=1e-12)
    assert list(dit.rope_frequencies(8, 10000.0, 2.0, 1e5, 1e300, 1e300)) == pytest.approx([0.5, 0.05, 0.005, 0.0005], rel=1e-14)
    # equal limits: a step
    assert list(dit.rope_frequencies(8, 10000.0, 2.0, 1e5, 200.0, 200.0)) == pytest.approx([1.0, 0.1, 0.005, 0.0005], rel=1e-14)
    assert len(dit.rope_frequencies(2, 5.0)) == 1 and len(dit.rope_frequencies(256, 5.0)) == 128


def test_rope_frequencies_refusals():
    bad = _refusals(dit.rope_frequencies, [8, 1e4, 2.0, 100.0, 1.0, 4.0])
    assert bad((0, 0)) == BAD and bad((0, 7)) == BAD and bad((0, -2)) == BAD and bad((0, 258)) == UNS
    for i, values in ((1, (0.0, -1.0, INF, NAN)), (2, (0.5, INF, NAN)), (3, (0.0, INF, NAN)), (4, (-1.0, 5.0, NAN)), (5, (NAN, 0.5))):
        for v in values:
            assert bad((i, v)) == BAD, (i, v)


def test_rope_refusals():
    w = dit.rope_frequencies(32, 1e4)
    bad = _refusals(dit.dit_rope, [5, 3, 64, 32, dit.DIT_ROPE_HALF, BF, P, w, 1.0, P, 192, P, 192, 0])
    assert bad((0, -1)) == BAD and bad((1, 0)) == BAD and bad((2, 0)) == BAD
    assert bad((3, 0)) == BAD and bad((3, 31)) == BAD and bad((2, 16), (10, 192)) == BAD
    assert bad((1, 1), (2, 2048), (10, 2048), (12, 2048)) == UNS
    assert _err(dit.dit_rope, 5, 1, 512, 258, 0, BF, P, [0.1] * 129, 1.0, P, 512, P, 512, 0) == UNS
    assert bad((4, 2)) == BAD and bad((5, 3)) == BAD and bad((7, None)) == BAD
    assert bad((7, [0.1] * 15 + [INF])) == BAD and bad((7, [NAN] * 16)) == BAD and bad((8, NAN)) == BAD and bad((8, INF)) == BAD
    assert bad((7, [0.1] * 15 + [1e300])) == BAD and bad((7, [-2.0 ** 65] + [0.1] * 15)) == BAD  # angles past a double's range
    assert bad((10, 191)) == BAD and bad((12, 191)) == BAD
    assert bad((9, 0)) == BAD and bad((11, 0)) == BAD and bad((9, P + 1)) == BAD and bad((11, P + 1)) == BAD and bad((6, P + 2)) == BAD
    assert bad((12, 200)) == BAD  # in place with another stride
    dit.dit_rope(0, 3, 64, 32, 0, BF, None, w, 1.0, 0, 192, 0, 192, 0)
    with pytest.raises(ValueError):
        dit.dit_rope(5, 3, 64, 32, 0, BF, P, [0.1] * 15, 1.0, P, 192, P, 192, 0)


def test_sequences_need_one_entry_each():
    with pytest.raises(ValueError):
        dit.Sequences([1, 2], [3])
    with pytest.raises(ValueError):
        dit.Sequences([1], [3], [0, 1])


def test_grouped_refusals():
    q = dit.Sequences([7, 1], [7, 40])
    size = dit.attention_grouped_workspace_size
    assert size(q, 6, 3, 64, BF) >= 0
    ok = [q, 6, 3, 64, BF, dit.DIT_CAUSAL, 0.125, P, 768, P, P, 768, P, 384, P, 1 << 40, 0]
    bad = _refusals(dit.dit_attention_grouped, ok)
    for fn in (lambda s: bad((0, s)), lambda s: _err(size, s, 6, 3, 64, BF)):
        assert fn(dit.Sequences([], [])) == BAD
        assert fn(dit.Sequences([1] * 129, [1] * 129)) == BAD
        assert fn(dit.Sequences([-1], [1])) == BAD and fn(dit.Sequences([1], [-1])) == BAD
        assert fn(dit.Sequences([1], [1], [-1])) == BAD and fn(dit.Sequences([1], [1], [(1 << 40) + 1])) == UNS
        assert fn(dit.Sequences([1], [(1 << 24) + 1])) == UNS
        assert fn(dit.Sequences([(1 << 24), 1], [1, 1])) == UNS
    for fn in (lambda *c: bad(*c), lambda *c: _refusals(size, ok[:5])(*c)):
        assert fn((1, 0)) == BAD and fn((2, 0)) == BAD and fn((2, 4)) == BAD and fn((1, 1026), (2, 1)) == UNS
        assert fn((3, 96)) == UNS and fn((4, 2)) == BAD and fn((3, 128), (4, F32)) == UNS
    # 2^21 queries of 1024 heads to one key head
    many = dit.Sequences([1 << 21], [1])
    assert _err(size, many, 1024, 1, 64, BF) == UNS and size(many, 1024, 1024, 64, BF) >= 0
    assert _err(dit.dit_attention_grouped, many, 1024, 1, 64, BF, 0, 0.125, P, 65536, P, P, 64, P, 65536, P, 1 << 40, 0) == UNS
    assert bad((5, 2)) == BAD and all(bad((6, v)) == BAD for v in (NAN, INF, 0.0, -1.0, 1e-20, 1e20))
    for i in (7, 9, 10, 12):
        assert bad((i, 0)) == BAD and bad((i, P + 8)) == BAD
    assert bad((8, 376)) == BAD and bad((11, 184)) == BAD and bad((13, 376)) == BAD
    assert bad((8, 772)) == BAD and bad((11, 388)) == BAD and bad((13, 388)) == BAD
    assert bad((8, (1 << 22) + 8)) == UNS and bad((11, (1 << 22) + 8)) == UNS and bad((13, (1 << 22) + 8)) == UNS
    assert bad((12, P)) == BAD  # o is q with another stride


def test_grouped_without_queries():
    """Nothing to do, and no pointer needed (that of a tensor without elements is NULL); the rest is checked as ever."""
    for dtype in (BF, F32):
        for q in (dit.Sequences([0], [0]), dit.Sequences([0, 0], [3000, 7]), dit.Sequences([0], [5], [9])):
            assert dit.attention_grouped_workspace_size(q, 6, 3, 64, dtype) == 0
            ok = [q, 6, 3, 64, dtype, dit.DIT_CAUSAL, 0.125, 0, 384, 0, 0, 192, 0, 384, 0, 0, 0]
            dit.dit_attention_grouped(*ok)
            bad = _refusals(dit.dit_attention_grouped, ok)
            assert bad((2, 4)) == BAD and bad((3, 96)) == UNS and bad((5, 2)) == BAD and bad((6, NAN)) == BAD
            assert bad((8, 376)) == BAD and bad((11, 184)) == BAD and bad((13, 376)) == BAD and bad((8, (1 << 22) + 8)) == UNS


def test_grouped_with_queries_needs_its_pointers():
    # keys of a sequence without queries are not read: with queries of the other, which has none, k and v may be NULL, q and o may not
    q = dit.Sequences([0, 3], [40, 0])
    ok = [q, 6, 3, 64, BF, 0, 0.125, P, 384, 0, 0, 192, P, 384, 0, 0, 0]
    bad = _refusals(dit.dit_attention_grouped, ok)
    assert bad((7, 0)) == BAD and bad((12, 0)) == BAD and bad((7, P + 8)) == BAD and bad((12, P + 8)) == BAD
    for seqs in (dit.Sequences([3], [1]), dit.Sequences([3, 3], [0, 1])):
        assert bad((0, seqs)) == BAD and bad((0, seqs), (9, P)) == BAD and bad((0, seqs), (10, P)) == BAD


def test_a_factor_needs_the_context_that_it_extends():
    """A factor without the length and the limits that say which pairs it divides would leave all frequencies as they are."""
    for args in ((2.0,), (2.0, 1e5), (2.0, 1e5, 1.0), (NAN,), (0.5,)):
        with pytest.raises(ValueError):
            dit.rope_frequencies(8, 1e4, *args)
    for kw in ({"low": 1.0, "high": 4.0}, {"original_len": 1e5, "high": 4.0}, {"original_len": 1e5, "low": 1.0}):
        with pytest.raises(ValueError):
            dit.rope_frequencies(8, 1e4, factor=8.0, **kw)
    plain = list(dit.rope_frequencies(8, 1e4))
    assert plain == list(dit.rope_frequencies(8, 1e4, 1.0)) == list(dit.rope_frequencies(8, 1e4, 1.0, 4096.0, 1.0, 4.0))
    assert plain == list(dit.rope_frequencies(8, 1e4, original_len=4096.0)) == list(dit.rope_frequencies(8, 1e4, low=1.0, high=4.0))
    assert list(dit.rope_frequencies(8, 1e4, 8.0, 1e5, low=0.0, high=0.0)) == plain  # asked for: every pair turns 0 times or more
    # limits that are given are checked without a factor too
    assert _err(dit.rope_frequencies, 8, 1e4, 1.0, 4096.0, 4.0, 1.0) == BAD
    assert _err(lambda: dit.rope_frequencies(8, 1e4, low=-1.0)) == BAD and _err(lambda: dit.rope_frequencies(8, 1e4, original_len=0.0)) == BAD


def test_grouped_workspace_is_of_these_lengths_and_bounded():
    size = dit.attention_grouped_workspace_size
    # one token over a cache of 32 / 8 heads of 128: ranges of 256 keys up to 16384, evenly longer ones from there on.  A
    # range of a key head holds 32 rows of 128 sums, a maximum and a sum.
    for keys, ranges in ((768, 0), (769, 4), (4096, 16), (16384, 64), (16385, 65), (16448, 52), (65536, 64), (1 << 24, 64)):
        assert size(dit.Sequences([1], [keys]), 32, 8, 128, BF) == ranges * 8 * 32 * 130 * 4, keys
    rng = random.Random(3)
    most = 0
    for _ in range(400):
        kv_heads = rng.choice([1, 2, 8, 32, 64, 128, 1024])
        heads = kv_heads * rng.choice([g for g in (1, 2, 8, 64) if g * kv_heads <= 1024])
        kv = [int(2 ** rng.uniform(0, 24)) for _ in range(rng.choice([1, 3, 30, 128]))]
        q = [min(m, int(2 ** rng.uniform(0, rng.choice([1, 6, 16])))) for m in kv]
        for d, dtype in ((64, BF), (128, BF), (64, F32)):
            most = max(most, size(dit.Sequences(q, kv), heads, kv_heads, d, dtype))
    assert 64 << 20 < most <= 128 << 20
