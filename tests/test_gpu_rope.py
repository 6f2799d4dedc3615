"""Rotary positions on the GPU against the fp64 reference.

Tolerance.  Sine and cosine of the angle, formed in 64 bits: off by at most 2^-22 in fp32 (what is left of the turns is
rounded to fp32, 2^-25 of a turn, and two steps of the functions), and by the angle's own rounding, 2^-51 of it, on either
side.  The products and their sum are rounded to fp32, times the magnitude: 2^-22 more of |a| + |b|.  bf16 output: half a
step (2^-8 of the value) more."""
import numpy as np
import pytest

from oracle import text_oracle as T
from paper_2510_01565_amd import dit, synth

pytestmark = pytest.mark.gpu
LAYOUT = {"half": dit.DIT_ROPE_HALF, "pairs": dit.DIT_ROPE_PAIRS}


def _torch():
    import torch
    return torch


def _check(got, x, pos, w, layout, magnitude, dtype):
    want = T.rope(x, pos, w, layout, magnitude)
    n = len(w)
    ia, ib = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    both = abs(magnitude) * (np.abs(x[:, :, ia]) + np.abs(x[:, :, ib]))
    off = 2.0 ** -21 + 2.0 ** -51 * np.abs(np.outer(pos, w))[:, None, :]
    tol = np.zeros(x.shape)
    tol[:, :, ia] = tol[:, :, ib] = both * off
    if dtype == "bf16":
        tol[:, :, :2 * n] += 2.0 ** -8 * np.abs(want[:, :, :2 * n])
    assert np.isfinite(got).all()
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - want).max())


def _run(rows, heads, d, rot, layout, dtype, pos, w, magnitude, gap_x=0, gap_y=0, inplace=False, shift=0, seed=0):
    torch = _torch()
    dt, code = (torch.bfloat16, dit.DIT_BF16) if dtype == "bf16" else (torch.float32, dit.DIT_F32)
    ldx, ldy = heads * d + gap_x, heads * d + (gap_x if inplace else gap_y)
    x = torch.from_numpy(synth.normal(seed, "x", (rows, ldx))).to(dt)
    flat = torch.zeros(rows * ldx + shift + 8, dtype=dt, device="cuda")
    flat[shift:shift + rows * ldx] = x.reshape(-1).cuda()
    out = flat if inplace else torch.full((rows * ldy + shift + 8,), 5.0, dtype=dt, device="cuda")
    dp = None if pos is None else torch.tensor(pos, dtype=torch.int32, device="cuda")
    dit.dit_rope(rows, heads, d, rot, LAYOUT[layout], code, dp, w, magnitude, flat[shift:], ldx, out[shift:], ldy)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    body = got[shift:shift + rows * ldy].reshape(rows, ldy)
    xs = x.double().numpy()
    if inplace:
        assert np.array_equal(body[:, heads * d:], xs[:, heads * d:])
    else:
        assert (got[:shift] == 5).all() and (got[shift + rows * ldy:] == 5).all() and (body[:, heads * d:] == 5).all()
        assert np.array_equal(flat[shift:shift + rows * ldx].double().cpu().numpy(), xs.reshape(-1))
    xs = xs[:, :heads * d].reshape(rows, heads, d)
    body = body[:, :heads * d].reshape(rows, heads, d)
    assert np.array_equal(body[:, :, rot:], xs[:, :, rot:])
    _check(body, xs, np.arange(rows) if pos is None else np.asarray(pos, np.float64), list(w), layout, magnitude, dtype)


CASES = [(1, 1, 64, 64), (1, 40, 128, 128), (3, 5, 64, 32), (7, 3, 80, 40), (2, 2, 96, 96), (5, 1, 10, 6), (4, 3, 33, 2), (130, 8, 128, 64),
         (9, 2, 256, 256), (6, 2, 320, 200), (2, 65, 64, 64), (3, 1, 1024, 16), (300, 6, 64, 48)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rows,heads,d,rot", CASES)
def test_rope(rows, heads, d, rot, layout, dtype):
    rng = np.random.default_rng(rows + d)
    pos = rng.integers(0, 100000, rows)
    w = dit.rope_frequencies(rot, 10000.0, 8.0, 4096.0, 1.0, 4.0)
    _run(rows, heads, d, rot, layout, dtype, pos, w, 1.2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("d,rot,gap,shift", [(64, 64, 0, 0), (64, 32, 192, 0), (128, 128, 8, 0), (64, 64, 7, 1), (128, 64, 3, 3), (24, 20, 5, 1)])
def test_in_place_strides_and_alignment(d, rot, gap, shift, layout, dtype):
    w = dit.rope_frequencies(rot, 500.0)
    _run(21, 3, d, rot, layout, dtype, None, w, 1.0, gap_x=gap, inplace=True, shift=shift)
    _run(21, 3, d, rot, layout, dtype, None, w, -0.5, gap_x=gap, gap_y=2 * gap, shift=shift)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_positions_of_every_size(layout):
    pos = [0, 1, -1, 2, 131071, 1 << 20, -(1 << 20), (1 << 31) - 1, -(1 << 31), 16777217]
    _run(len(pos), 4, 128, 128, layout, "f32", pos, dit.rope_frequencies(128, 10000.0), 1.0)
    _run(len(pos), 4, 128, 128, layout, "f32", pos, [0.0, 1e-9, -3.0, 6.283185307179586] * 16, 1.0)


def test_many_rows_and_many_heads():
    w = dit.rope_frequencies(32, 10000.0)
    _run(5000, 3, 32, 32, "half", "bf16", None, w, 1.0)
    _run(2, 3000, 32, 32, "pairs", "f32", None, w, 1.0)


def test_not_finite_values_stay_in_their_pair():
    torch = _torch()
    x = torch.ones((2, 2, 64), dtype=torch.float32, device="cuda")
    x[1, 0, 3], x[0, 1, 40], x[0, 0, 63] = float("nan"), float("inf"), float("nan")
    for layout in ("half", "pairs"):
        y = torch.empty_like(x)
        dit.dit_rope(2, 2, 64, 48, LAYOUT[layout], dit.DIT_F32, None, dit.rope_frequencies(48, 100.0), 1.0, x, 128, y, 128)
        fin = torch.isfinite(y).cpu()
        want = torch.ones_like(fin)
        a, b = ((3, 27), (40, 16)) if layout == "half" else ((2, 3), (40, 41))
        want[1, 0, list(a)] = False
        want[0, 1, list(b)] = False
        want[0, 0, 63] = False
        assert torch.equal(fin, want)


def test_captured():
    torch = _torch()
    x = torch.randn((33, 4 * 64), device="cuda")
    pos = torch.arange(33, dtype=torch.int32, device="cuda")
    w = dit.rope_frequencies(64, 10000.0)
    y = torch.empty_like(x)
    call = lambda: dit.dit_rope(33, 4, 64, 64, dit.DIT_ROPE_HALF, dit.DIT_F32, pos, w, 1.0, x, 256, y, 256)
    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for step in range(3):
        pos += 7
        call()
        torch.cuda.synchronize()
        want = y.clone()
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
