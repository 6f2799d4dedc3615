"""Pins of the reference of the 8-bit products and the block-sparse attention
(CPU): hand values, torch's own conversion, and the dense attention."""
import numpy as np
import pytest
import torch

import oracle as O
from oracle import lowbit_oracle as B


def test_e4m3_values_are_those_of_torch():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    v = B.e4m3_values()
    assert np.array_equal(v, t, equal_nan=True)
    assert v[0x7e] == 448 and v[0x38] == 1 and v[1] == 2.0 ** -9 and np.isnan(v[0x7f])


def test_e4m3_encode_rounds_to_nearest_even():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=20000) * np.exp(3 * rng.normal(size=20000)), [448, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10]])
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(B.e4m3_encode(x.astype(np.float64)), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    # ties: between 1 and 1.125, 1.125 and 1.25; half of the smallest value goes to 0, one and a half of it to twice
    assert list(B.e4m3_values()[B.e4m3_encode(np.array([1.0625, 1.1875, 2.0 ** -10, 1.5 * 2.0 ** -9]))]) == [1.0, 1.25, 0.0, 2.0 ** -8]


@pytest.mark.parametrize("a,e", [(448.0, 0), (448.0001, 1), (1.75, -8), (1.7500001, -7), (2.0, -7), (1e-45, -127), (0.0, 0)])
def test_scale_is_the_smallest_power_of_two(a, e):
    assert B.scale_exponent(a) == e


def test_quantize_pads_and_keeps_non_finite_values_out_of_the_scale():
    x = np.zeros((3, 130))
    x[0, 0], x[0, 1], x[1, 128], x[2, 129] = 3.5, np.inf, np.nan, -896
    q, s = B.quantize_fp8(x, 1)
    assert q.shape == (3, 256) and s.shape == (3, 4)
    assert s[0, 0] == 127 - 7 and B.e4m3_values()[q[0, 0]] == 448 and q[0, 1] == 0x7f
    assert s[1, 1] == 127 and q[1, 128] == 0x7f and s[2, 1] == 128 and B.e4m3_values()[q[2, 129]] == -448
    assert not q[:, 130:].any() and (s[:, 2:] == 127).all()
    q, s = B.quantize_fp8(x, 128)
    assert s.shape == (1, 4) and s[0, 1] == 128
    d = B.dequantize_fp8(q, s, 128, 130)
    assert d[2, 129] == -896 and np.isnan(d[1, 128])


def test_select_ranks_text_then_nan_then_score():
    q = np.ones((128, 1, 4))
    k = np.zeros((64 * 5 + 3, 1, 4))
    for j, x in enumerate((1.0, 5.0, 5.0, 7.0, 2.0, 9.0)):
        k[j * 64:(j + 1) * 64] = x
    q = np.ones((k.shape[0], 1, 4))
    assert B.select_blocks(q, k, 2)[0, 0].tolist() == [3, 5]
    assert B.select_blocks(q, k, 3)[0, 0].tolist() == [1, 3, 5]          # of the two equal ones the lower index
    assert B.select_blocks(q, k, 2, n_text=65)[0, 2].tolist() == [0, 1]
    assert B.select_blocks(q, k, 8)[0, 0].tolist() == [0, 1, 2, 3, 4, 5, -1, -1]
    k[0, 0, 0] = np.nan
    assert B.select_blocks(q, k, 2)[0, 0].tolist() == [0, 5]


def test_sparse_attention_over_all_blocks_is_the_dense_one():
    rng = np.random.default_rng(1)
    q, k, v = (rng.normal(size=(150, 2, 8)) for _ in range(3))
    blocks = np.array([[[2, 0, 1, 1], [0, 1, 2, -1]]] * 2)
    o = B.sparse_attention(q, k, v, blocks)
    assert np.abs(o - O.attention(q, k, v)).max() < 1e-12
    # a listed block alone, an empty list, entries out of range
    blocks = np.array([[[2, 7, -5, 2], [-1, 3, 1 << 30, -(1 << 31)]]] * 2)
    o = B.sparse_attention(q, k, v, blocks)
    assert np.abs(o[:128] - O.attention(np.concatenate([q[:128], k[128:]]), np.concatenate([k[128:]]), v[128:])[:128]).max() < 1e-12
    assert not o[128:].any()
