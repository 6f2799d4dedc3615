"""The reference of the 4-bit matrices, the rotary positions and the grouped attention against hand-worked values."""
import numpy as np
import torch

from oracle import text_oracle as T


def test_e2m1_rounding():
    v = [0.0, 0.24, 0.25, 0.26, 0.74, 0.75, 0.76, 1.25, 1.26, 1.75, 2.5, 2.51, 3.5, 5.0, 5.01, 6.0, -0.3, -6.0]
    want = [0, 0, 0, 0.5, 0.5, 1, 1, 1, 1.5, 2, 2, 3, 4, 4, 6, 6, 0.5, 6]
    assert T.E2M1[T.round_e2m1(v)].tolist() == want


def test_scales_are_the_smallest_that_hold_a_block():
    x = np.zeros((1, 7 * 32))
    for b, a in enumerate([6.0, 6.0001, 12.0, 1.0, 2.0 ** -140, 1.5, 0.75 * 2.0 ** 127]):
        x[0, b * 32 + 5] = -a
    _, s = T.quantize_fp4(x)
    got = [int(s[0, T.scale_place(b)]) - 127 for b in range(7)]
    assert got == [0, 1, 1, -2, -127, -2, 124]
    assert s.shape == (1, 16) and (np.delete(s[0], [T.scale_place(b) for b in range(7)]) == 127).all()


def test_codes_places_and_way_back():
    x = np.zeros((2, 300))
    x[0, 0], x[0, 1], x[0, 299], x[1, 33] = 6, -1, 3, 0.5
    q, s = T.quantize_fp4(x)
    assert q.shape == (2, 256) and s.shape == (2, 16)
    assert q[0, 0] == 7 | (8 + 2) << 4                     # 6 and -1
    assert q[0, 149] == 7 << 4 and s[0, T.scale_place(9)] == 126  # 3 = 6 * 2^-1
    assert q[1, 16] == 6 << 4 and s[1, T.scale_place(1)] == 127 - 3  # 0.5 = 4 * 2^-3
    assert T.scale_place(9) == 6 and T.scale_place(4) == 1 and T.scale_place(17) == 20
    assert np.array_equal(T.dequantize_fp4(q, s, 300), x)


def test_a_value_that_is_not_finite_makes_its_block_nan():
    x = np.ones((1, 96))
    x[0, 40] = np.inf
    q, s = T.quantize_fp4(x)
    back = T.dequantize_fp4(q, s, 96)
    assert np.isnan(back[0, 32:64]).all() and (back[0, :32] == 1).all() and (back[0, 64:] == 1).all()


def test_rope_is_a_turn_of_complex_numbers():
    rng = np.random.default_rng(0)
    x, pos, w = rng.normal(size=(4, 2, 10)), [0, 1, -3, 70000], [1.0, 0.1, 1e-3]
    for layout, at in (("half", ([0, 1, 2], [3, 4, 5])), ("pairs", ([0, 2, 4], [1, 3, 5]))):
        y = T.rope(x, pos, w, layout, 1.25)
        z = (x[:, :, at[0]] + 1j * x[:, :, at[1]]) * 1.25 * np.exp(1j * np.outer(pos, w))[:, None]
        assert np.allclose(y[:, :, at[0]], z.real) and np.allclose(y[:, :, at[1]], z.imag)
        assert np.array_equal(y[:, :, 6:], x[:, :, 6:])


def test_grouped_attention_against_torch():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(5, 6, 8)), rng.normal(size=(9, 2, 8)), rng.normal(size=(9, 2, 8))
    o, _ = T.grouped_attention(q, k, v, [2, 0, 3], [4, 2, 3], [5, 0, 1], 0.3, True)
    for at, n, f, m in ((0, 2, 5, 4), (2, 3, 1, 3)):
        mask = torch.arange(m)[None] <= torch.arange(m - n, m)[:, None]
        qt, kt, vt = (torch.from_numpy(np.ascontiguousarray(t)).transpose(0, 1) for t in (q[at:at + n], k[f:f + m], v[f:f + m]))
        ref = torch.nn.functional.scaled_dot_product_attention(qt[None], kt.repeat_interleave(3, 0)[None],
                                                               vt.repeat_interleave(3, 0)[None], attn_mask=mask, scale=0.3)
        assert np.allclose(o[at:at + n], ref[0].transpose(0, 1).numpy())


def test_queries_before_the_first_key_get_zero():
    o, _ = T.grouped_attention(np.ones((3, 1, 4)), np.ones((1, 1, 4)), 7 * np.ones((1, 1, 4)), [3], [1], [0], 1.0, True)
    assert o[:, 0, 0].tolist() == [0, 0, 7]
