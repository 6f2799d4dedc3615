"""Quantising to e2m1, back, and the products of 4-bit matrices on the GPU, against the fp64 reference.

Tolerances.  Codes, scales and values: equal.  fp32 output: of each 8 products, which share their scales, the sum is
exact; every addition of such a sum loses less than one step of fp32 (2^-23, whether it rounds or cuts) of the products'
magnitudes, and the bias one more: (K / 8 + 2) 2^-23 of them.  bf16 output: half a step (2^-8 of the value) more."""
import math

import numpy as np
import pytest

from oracle import text_oracle as T
from paper_2510_01565_amd import dit, synth

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _dt(name):
    torch = _torch()
    return (torch.bfloat16, dit.DIT_BF16) if name == "bf16" else (torch.float32, dit.DIT_F32)


def _guarded(n):
    """n bytes between two runs of 0xa5: the buffer and a check that nothing around it was written."""
    torch = _torch()
    t = torch.full((n + 512,), 0xa5, dtype=torch.uint8, device="cuda")
    return t[256:256 + n], lambda: bool((t[:256] == 0xa5).all() and (t[256 + n:] == 0xa5).all())


def _quantize(x, rows, K, dtype):
    nc, ns = dit.fp4_layout(rows, K)
    q, okq = _guarded(nc)
    s, oks = _guarded(ns)
    dit.dit_quantize_fp4(rows, K, dtype, x, q, s)
    _torch().cuda.synchronize()
    assert okq() and oks()
    return q.cpu().numpy().reshape(rows, -1), s.cpu().numpy().reshape(rows, -1), q, s


def _matrix(seed, rows, K, bf16):
    """Normal values of widely differing rows and blocks, with zeros, an empty block and values far below their block's largest."""
    x = synth.normal(seed, "x", (rows, K))
    rng = np.random.default_rng(seed)
    x *= np.exp(2 * rng.normal(size=(rows, 1))).astype(np.float32)
    for j in range(0, K, 32):
        x[:, j:j + 32] *= np.float32(2.0 ** rng.integers(-12, 12))
    x[rng.random(x.shape) < 0.05] = 0
    x[rng.random(x.shape) < 0.02] *= np.float32(2.0 ** -6)
    if K > 64:
        x[:, 32:64] = 0
    t = _torch().from_numpy(x)
    return t.to(_torch().bfloat16) if bf16 else t


QSHAPES = [(1, 1), (1, 32), (2, 33), (3, 7), (5, 255), (4, 256), (4, 257), (6, 511), (3, 512), (2, 513), (130, 100), (9, 1537)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K", QSHAPES)
def test_quantize_and_back(rows, K, dtype):
    torch = _torch()
    x = _matrix(rows * 7 + K, rows, K, dtype == "bf16")
    q, s, dq, ds = _quantize(x.cuda(), rows, K, _dt(dtype)[1])
    rq, rs = T.quantize_fp4(x.double().numpy())
    assert np.array_equal(s, rs)
    assert np.array_equal(q, rq)
    want = T.dequantize_fp4(q, s, K)
    for out in ("bf16", "f32"):
        es = 2 if out == "bf16" else 4
        y, ok = _guarded(rows * K * es)
        dit.dit_dequantize_fp4(rows, K, dq, ds, _dt(out)[1], y)
        torch.cuda.synchronize()
        assert ok()
        assert np.array_equal(y.view(_dt(out)[0]).double().cpu().numpy().reshape(rows, K), want)


@pytest.mark.parametrize("shift", [1, 3])
@pytest.mark.parametrize("K", [64, 200])
def test_unaligned_rows(shift, K):
    """x, and the values on their way back, anywhere their elements may lie."""
    torch = _torch()
    x = _matrix(K + shift, 40, K, True)
    big = torch.zeros(40 * K + 8, dtype=torch.bfloat16, device="cuda")
    big[shift:shift + 40 * K] = x.reshape(-1).cuda()
    q, s, dq, ds = _quantize(big[shift:], 40, K, dit.DIT_BF16)
    rq, rs = T.quantize_fp4(x.double().numpy())
    assert np.array_equal(s, rs) and np.array_equal(q, rq)
    y = torch.full((40 * K + 8,), 9.0, dtype=torch.bfloat16, device="cuda")
    dit.dit_dequantize_fp4(40, K, dq, ds, dit.DIT_BF16, y[shift:])
    got = y.double().cpu().numpy()
    assert np.array_equal(got[shift:shift + 40 * K].reshape(40, K), T.dequantize_fp4(q, s, K))
    assert (got[:shift] == 9).all() and (got[shift + 40 * K:] == 9).all()


def test_extreme_values():
    """Infinities, NaN, the type's extremes and subnormals, ties, exact limits of a scale, signed zeros."""
    torch = _torch()
    x = torch.zeros((8, 96), dtype=torch.float32)
    x[0, :3] = torch.tensor([1.0, float("inf"), 2.0])
    x[1, 40] = float("nan")
    x[2, 70] = -float("inf")
    x[3, :2] = torch.tensor([3.4028234e38, 1e30])
    x[3, 32:34] = torch.tensor([1e-45, -1.2e-38])
    x[4, :17] = torch.tensor([6.0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, -.25, -.75, -5.0, .24999999, .25000003, 4.9999995, 5.0000005, -0.0, 0.0])
    x[5, :2] = torch.tensor([6.0000005, 1.0])
    x[6, 32:35] = torch.tensor([2.0 ** -127, 2.0 ** -126 * 1.5, 2.0 ** -149])
    x[7, 64:66] = torch.tensor([1.5 * 2.0 ** 127, -2.0 ** 127])
    q, s, dq, ds = _quantize(x.cuda(), 8, 96, dit.DIT_F32)
    rq, rs = T.quantize_fp4(x.double().numpy())
    assert np.array_equal(s, rs) and np.array_equal(q, rq)
    want = T.dequantize_fp4(q, s, 96)
    for out in ("bf16", "f32"):
        y = torch.empty((8, 96), dtype=_dt(out)[0], device="cuda")
        dit.dit_dequantize_fp4(8, 96, dq, ds, _dt(out)[1], y)
        got = y.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        top = float(torch.finfo(_dt(out)[0]).max)
        want_out = np.where(np.abs(want) > top, np.sign(want) * np.inf, want)
        ok = ~np.isnan(want)
        assert np.array_equal(got[ok], want_out[ok])
    assert np.isnan(want[0, :32]).all() and np.isnan(want[1, 32:64]).all() and np.isnan(want[2, 64:]).all()


def _product(M, N, K, out, bias, seed, noise=None):
    """Operands, the call's output, and the exact product with the sum of magnitudes."""
    torch = _torch()
    x = _matrix(seed, M, K, True)
    w = torch.from_numpy(synth.normal(seed, "w", (N, K), std=0.02)).to(torch.bfloat16)
    if noise is not None:
        noise(x, w)
    xq, xs, dxq, dxs = _quantize(x.cuda(), M, K, dit.DIT_BF16)
    wq, ws, dwq, dws = _quantize(w.cuda(), N, K, dit.DIT_BF16)
    b = None if bias is None else torch.from_numpy(synth.normal(seed, "b", (N,))).to(_dt(bias)[0])
    y = torch.full((M * N + 8,), float("nan"), dtype=_dt(out)[0], device="cuda")
    dit.dit_linear_fp4(M, N, K, dxq, dxs, dwq, dws, None if b is None else b.cuda(), _dt(bias or "bf16")[1], y, _dt(out)[1])
    torch.cuda.synchronize()
    assert torch.isnan(y[M * N:]).all()  # nothing behind the last row
    xv, wv = T.dequantize_fp4(xq, xs, K), T.dequantize_fp4(wq, ws, K)
    ref, mag = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    if b is not None:
        ref, mag = ref + b.double().numpy(), mag + np.abs(b.double().numpy())
    return y[:M * N].double().cpu().numpy().reshape(M, N), ref, mag


def _check(got, ref, mag, K, out):
    tol = (K / 8 + 2) * 2.0 ** -23 * mag
    if out == "bf16":
        tol = tol + 2.0 ** -8 * np.abs(ref)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) / tol).max()
    err = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    assert err < (2.0 ** -8 if out == "bf16" else 4 * K ** 0.5 * 2.0 ** -24), err


SHAPES = [(1, 1, 1), (1, 3001, 64), (1, 130, 4096), (4, 9216, 384), (15, 33, 700), (16, 256, 128), (17, 100, 1536), (33, 1000, 250),
          (64, 64, 6144), (65, 130, 129), (128, 128, 512), (129, 200, 640), (200, 511, 300), (333, 1024, 1536),
          (577, 700, 1000), (1030, 2050, 390), (260, 300, 1100), (300, 2304, 2560)]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear_fp4(M, N, K, out):
    bias = {0: None, 1: "bf16", 2: "f32"}[(M + N) % 3]
    got, ref, mag = _product(M, N, K, out, bias, M + N + K)
    _check(got, ref, mag, K, out)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(2, 40, 300), (40, 70, 300), (300, 300, 300), (600, 520, 800), (3500, 3490, 1700)])
def test_a_nan_reaches_its_row_alone(M, N, K, out):
    """A NaN or an infinity of x makes its own output row NaN, one of w its own column."""
    def noise(x, w):
        x[1, 5] = float("inf")
        w[7, K - 1] = float("nan")
    got, ref, _ = _product(M, N, K, out, "f32", 3, noise)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    assert np.isnan(ref).sum() == N + M - 1


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(3, 260), (50, 260), (400, 260), (8150, 4090)])
def test_scales_of_every_size(M, N, out):
    """Blocks whose scales lie 2^100 apart on either side, all powers passing through the same output."""
    def noise(x, w):
        for j in range(0, x.shape[1], 32):
            e = (j // 32) * 3 - 50
            x[:, j:j + 32] = (x[:, j:j + 32].float() * 2.0 ** e).to(x.dtype)
            w[:, j:j + 32] = (w[:, j:j + 32].float() * 2.0 ** -e).to(w.dtype)
    got, ref, mag = _product(M, N, 1100, out, None, 5, noise)
    _check(got, ref, mag, 1100, out)


@pytest.mark.parametrize("M,N,K", [(9, 300, 900), (70, 300, 900), (600, 700, 900), (3500, 3490, 1700)])
def test_rows_do_not_depend_on_other_rows_values(M, N, K):
    """Same M and N: a row's bits are its own, and equal on every call."""
    torch = _torch()
    x = _matrix(1, M, K, True)
    w = torch.from_numpy(synth.normal(1, "w", (N, K), std=0.02)).to(torch.bfloat16)
    outs = []
    for other in (0, 0, 1):
        if other:
            x[1:] = _matrix(2, M, K, True)[1:]
        _, _, xq, xs = _quantize(x.cuda(), M, K, dit.DIT_BF16)
        _, _, wq, ws = _quantize(w.cuda(), N, K, dit.DIT_BF16)
        y = torch.empty((M, N), dtype=torch.float32, device="cuda")
        dit.dit_linear_fp4(M, N, K, xq, xs, wq, ws, None, dit.DIT_BF16, y, dit.DIT_F32)
        outs.append(y.clone())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0][0], outs[2][0]) and not torch.equal(outs[0], outs[2])


def _large(M, N, K, out, bias, seed, off=0):
    """A product too large for the host: 64 bits on the GPU from the values that the codes stand for.  off: elements by
    which y is misaligned."""
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((M, K), generator=gen, device="cuda") * torch.exp(torch.randn((M, 1), generator=gen, device="cuda"))
    x *= torch.exp(2 * torch.randn((1, -(-K // 32)), generator=gen, device="cuda")).repeat_interleave(32, 1)[:, :K]
    w = torch.randn((N, K), generator=gen, device="cuda") * 0.02
    b = torch.randn((N,), generator=gen, device="cuda") if bias else None
    ops = []
    for t, rows in ((x, M), (w, N)):
        nc, ns = dit.fp4_layout(rows, K)
        q, s = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")
        dit.dit_quantize_fp4(rows, K, dit.DIT_F32, t, q, s)
        v = torch.empty((rows, K), dtype=torch.float32, device="cuda")
        dit.dit_dequantize_fp4(rows, K, q, s, dit.DIT_F32, v)
        ops.append((q, s, v))
    dt = _dt(out)[0]
    y = torch.full((M * N + off + 64,), 7.0, dtype=dt, device="cuda")
    dit.dit_linear_fp4(M, N, K, ops[0][0], ops[0][1], ops[1][0], ops[1][1], b, dit.DIT_F32, y[off:], _dt(out)[1])
    torch.cuda.synchronize()
    assert (y[:off] == 7).all() and (y[off + M * N:] == 7).all()
    y = y[off:off + M * N].view(M, N)
    wt = ops[1][2].double().t().contiguous()
    worst = 0.0
    for r in range(0, M, 4096):
        xv = ops[0][2][r:r + 4096].double()
        ref, mag = xv @ wt, xv.abs() @ wt.abs()
        if b is not None:
            ref, mag = ref + b.double(), mag + b.double().abs()
        tol = (K / 8 + 2) * 2.0 ** -23 * mag + (2.0 ** -8 * ref.abs() if out == "bf16" else 0.0)
        worst = max(worst, float(((y[r:r + 4096].double() - ref).abs() / tol).max()))
    assert worst <= 1.0, worst


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(16, 16384, 4096), (1, 20011, 4100), (100, 4096, 4096), (700, 3333, 2000), (4429, 1536, 1536),
                                   (2049, 2303, 777), (3500, 3490, 1700), (9000, 4500, 2000), (16717, 6150, 2000), (8190, 8190, 700), (5000, 6144, 1536), (4100, 8190, 1280), (8192, 4096, 512), (3000, 3000, 64)])
def test_linear_fp4_large(M, N, K, out):
    _large(M, N, K, out, (M + K) % 2 == 0, M + N)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K,off", [(3, 77, 200, 1), (90, 333, 300, 1), (2100, 2047, 900, 3), (4096, 4096, 1024, 1), (8190, 8190, 700, 3)])
def test_output_anywhere_its_elements_may_lie(M, N, K, off, out):
    _large(M, N, K, out, True, 11, off)


@pytest.mark.parametrize("bias", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(3, 77, 200), (40, 333, 1500), (200, 333, 300), (1030, 2050, 390), (3500, 3490, 1700)])
def test_bias_anywhere_its_elements_may_lie(M, N, K, bias):
    """A bias one element behind a 16-byte boundary gives the same bits as one at it."""
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(9)
    ops = []
    for rows in (M, N):
        t = torch.randn((rows, K), generator=gen, device="cuda")
        nc, ns = dit.fp4_layout(rows, K)
        ops += [torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")]
        dit.dit_quantize_fp4(rows, K, dit.DIT_F32, t, ops[-2], ops[-1])
    b = torch.randn(N, generator=gen, device="cuda").to(_dt(bias)[0])
    shifted = torch.cat([torch.full((1,), math.nan, device="cuda", dtype=b.dtype), b, torch.full((9,), math.nan, device="cuda", dtype=b.dtype)])
    outs = []
    for v in (b, shifted[1:], None):
        y = torch.empty((M, N), dtype=torch.float32, device="cuda")
        dit.dit_linear_fp4(M, N, K, *ops, v, _dt(bias)[1], y, dit.DIT_F32)
        outs.append(y)
    assert torch.equal(outs[0], outs[1])
    assert torch.isfinite(outs[0]).all() and torch.equal(outs[2] + b.float(), outs[0])


def test_one_long_row_and_one_long_column():
    _large(1, 1 << 18, 96, "bf16", False, 1)
    _large(1 << 18, 1, 96, "f32", True, 2)
    _large(2, 3, 1 << 20, "f32", False, 3)


def test_on_another_stream_and_captured():
    """Quantise and multiply on a side stream, then as a graph that is replayed with new inputs between."""
    torch = _torch()
    M, N, K = 48, 1024, 1536
    gen = torch.Generator(device="cuda").manual_seed(4)
    xs = [torch.randn((M, K), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3)]
    w = (torch.randn((N, K), generator=gen, device="cuda") * 0.02).to(torch.bfloat16)
    nc, ns = dit.fp4_layout(M, K)
    wc, wn = dit.fp4_layout(N, K)
    buf = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    q, s, wq, ws = buf(nc), buf(ns), buf(wc), buf(wn)
    x, y = torch.empty_like(xs[0]), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    dit.dit_quantize_fp4(N, K, dit.DIT_BF16, w, wq, ws)

    def layer():
        dit.dit_quantize_fp4(M, K, dit.DIT_BF16, x, q, s)
        dit.dit_linear_fp4(M, N, K, q, s, wq, ws, None, dit.DIT_BF16, y, dit.DIT_BF16)
    want = []
    for t in xs:
        x.copy_(t)
        layer()
        want.append(y.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.zero_()
        layer()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want[2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        layer()
    for rep in range(2):
        for t, r in zip(xs, want):
            x.copy_(t)
            y.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, r), rep


@pytest.mark.parametrize("M,N,K,kernel", [
    (16, 128, 1024, "rows"), (33, 1536, 6144, "16x32"), (128, 1536, 6144, "32x32"), (500, 1536, 1024, "64x64"),
    (1024, 4096, 1024, "128x128"), (4096, 8192, 1024, "256x256")])
def test_products_of_a_block_are_summed_exactly(M, N, K, kernel):
    """Each row one block that makes 2^24, where fp32 has steps of 2, ahead of or behind one whose products are +1 and -1 at
    random places and come to a positive even number: an output that is exact, which it would not be if fewer than all of a
    block's products, of which some come to an odd number, were added to the running sum at a time."""
    torch = _torch()
    rng = np.random.default_rng(M)
    blocks = K // 32
    codes, scales, want = np.zeros((M, K), np.uint8), np.full((M, blocks), 127, np.uint8), np.zeros(M)
    for m in range(M):
        big, small = rng.choice(blocks, 2, replace=False)
        codes[m, big * 32 + rng.integers(32)] = 6                  # 4, times 0.5 and 2^23
        scales[m, big] = 127 + 23
        minus = int(rng.integers(0, 8))
        plus = minus + 2 * int(rng.integers(1, 9))
        at = small * 32 + rng.permutation(32)[:plus + minus]
        codes[m, at[:plus]], codes[m, at[plus:]] = 2, 2 | 8       # 1 and -1, times 0.5 and 2
        scales[m, small] = 128
        sign = 8 * (m % 2)
        codes[m][codes[m] > 0] ^= sign
        want[m] = (2.0 ** 24 + plus - minus) * (-1) ** (m % 2)
    assert np.array_equal(want, want.astype(np.float32))
    spread = np.full((M, -(-blocks // 16) * 16), 127, np.uint8)
    spread[:, :blocks] = scales
    spread = spread.reshape(M, -1, 4, 4).transpose(0, 1, 3, 2).reshape(M, -1)
    nc, ns = dit.fp4_layout(M, K)
    packed = codes[:, 0::2] | codes[:, 1::2] << 4
    assert packed.size == nc and spread.size == ns
    xq, xs = (torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (packed, spread))
    assert np.array_equal(T.dequantize_fp4(packed, spread, K).sum(1) / 2, want)
    nc, ns = dit.fp4_layout(N, K)
    wq = torch.full((nc,), 0x11, dtype=torch.uint8, device="cuda")   # 0.5 everywhere
    ws = torch.full((ns,), 127, dtype=torch.uint8, device="cuda")
    y = torch.empty((M, N), dtype=torch.float32, device="cuda")
    dit.profile_start()
    dit.dit_linear_fp4(M, N, K, xq, xs, wq, ws, None, dit.DIT_BF16, y, dit.DIT_F32)
    assert set(dit.profile_stop()) == {"gemm_fp4_" + kernel}
    want = torch.from_numpy(want).float().cuda()
    wrong = (y != want[:, None]).nonzero()
    assert wrong.numel() == 0, (wrong.shape[0], [(int(m), float(y[m, n] - want[m])) for m, n in wrong[:4]])
