"""Block-sparse attention and the selection of its key blocks on the GPU, against
the fp64 reference.

Tolerances.  Lists: equal.  fp32 output: scores of 64 products and their scaling
are off by (64 + 3) 2^-24 of the magnitudes' sum S at most, which moves each
probability by as much relative to itself; the sums of n probabilities add
(n + 8) 2^-24.  bf16 output: besides that, each probability is rounded (2^-8 of it,
in the sum that divides too) and so is the output (2^-8): 3 * 2^-8.  All of it
relative to sum_j p_j |v_j|."""
import numpy as np
import pytest

from oracle import lowbit_oracle as B
from paper_2510_01565_amd import dit, synth

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 64), ("bf16", 128), ("f32", 64)]


def _torch():
    import torch
    return torch


def _dt(name):
    torch = _torch()
    return (torch.bfloat16, dit.DIT_BF16) if name == "bf16" else (torch.float32, dit.DIT_F32)


def _batch(reqs):
    """reqs: (grid_h, grid_w, n_txt) per request."""
    return dit.Batch([r[0] for r in reqs], [r[1] for r in reqs], [r[2] for r in reqs]), [r[0] * r[1] + r[2] for r in reqs]


def _qkv(seed, T, heads, d, dtype, gain=1.0):
    torch = _torch()
    out = []
    for n, g in (("q", gain ** 0.5), ("k", gain ** 0.5), ("v", 1.0)):
        out.append(torch.from_numpy(synth.normal(seed, n, (T, heads, d)) * np.float32(g)).to(_dt(dtype)[0]))
    return out


def _lists(seed, lens, heads, keep):
    """Random lists: unsorted, with repeats, entries out of range, empty ones and full ones."""
    rng = np.random.default_rng(seed)
    out = []
    for L in lens:
        n = -(-L // 64)
        a = rng.integers(-2, n + 2, size=(heads, -(-L // 128), keep))
        a[rng.random(a.shape) < 0.1] = np.iinfo(np.int32).max
        a[rng.random(a.shape) < 0.1] = np.iinfo(np.int32).min
        a[rng.random(a.shape[:2]) < 0.15] = -1                     # empty lists
        full = rng.random(a.shape[:2]) < 0.15
        a[full] = np.resize(np.arange(n), keep)
        out.append(a)
    return np.concatenate(out, 1).astype(np.int32)


def _run(b, heads, d, dtype, q, k, v, blocks, stream=None):
    """The call on buffers that go on past the last sequence; what lies there stays."""
    torch = _torch()
    T = q.shape[0]
    n = dit.attention_sparse_workspace_size(b, heads, d, _dt(dtype)[1])
    ws = torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")
    o = torch.full((T + 3, heads, d), 77.0, dtype=q.dtype, device="cuda")
    dit.dit_attention_sparse(b, heads, d, _dt(dtype)[1], q, k, v, blocks, blocks.shape[2], o, ws, n, stream)
    torch.cuda.synchronize()
    assert (o[T:] == 77).all()
    return o[:T]


def _check(o, q, k, v, blocks, lens, dtype):
    off = row = 0
    d = q.shape[2]
    for L in lens:
        nq, sl = -(-L // 128), slice(off, off + L)
        qq, kk, vv = (x[sl].double().numpy() for x in (q, k, v))
        ref, mag = B.sparse_attention(qq, kk, vv, blocks[:, row:row + nq], mag=True)
        got = o[sl].double().cpu().numpy()
        assert np.isfinite(got).all()
        S = max(np.abs(qq[:, h]).sum(1).max() * np.abs(kk[:, h]).max() for h in range(q.shape[1])) / d ** 0.5
        rel = 2 * (d + 3) * 2.0 ** -24 * S + (64 * blocks.shape[2] + 8) * 2.0 ** -24 + (3 * 2.0 ** -8 if dtype == "bf16" else 0)
        assert (np.abs(got - ref) <= rel * mag).all(), (np.abs(got - ref) / np.maximum(rel * mag, 1e-300)).max()
        assert not got[mag == 0].any()   # an empty list: exact zeros
        off += L
        row += nq


BATCHES = [
    ([(1, 1, 0)], 1), ([(1, 1, 0)], 3), ([(7, 9, 0)], 1), ([(8, 8, 0)], 2), ([(8, 8, 1)], 2), ([(1, 127, 0)], 2),
    ([(8, 16, 0)], 2), ([(8, 16, 1)], 3), ([(1, 1, 0), (5, 40, 57), (16, 16, 0), (1, 1, 2)], 3),
    ([(23, 23, 100)], 5), ([(32, 32, 333), (9, 9, 0)], 12),
]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("reqs,keep", BATCHES)
def test_sparse_attention(reqs, keep, dtype, d):
    torch = _torch()
    b, lens = _batch(reqs)
    heads = 3
    q, k, v = _qkv(sum(lens) + keep, sum(lens), heads, d, dtype)
    blocks = _lists(sum(lens), lens, heads, keep)
    o = _run(b, heads, d, dtype, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda())
    _check(o, q, k, v, blocks, lens, dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_sparse_attention_large_logits(dtype, d):
    """Scores of hundreds, their maxima far apart and in any block."""
    torch = _torch()
    b, lens = _batch([(20, 20, 39), (12, 12, 0)])
    q, k, v = _qkv(4, sum(lens), 2, d, dtype, gain=16.0)
    blocks = _lists(5, lens, 2, 4)
    o = _run(b, 2, d, dtype, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda())
    _check(o, q, k, v, blocks, lens, dtype)


@pytest.mark.parametrize("gain", [1.0, 16.0])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_lists_of_every_length_up_to_nine(dtype, d, gain):
    """Few query blocks with long lists of 0 .. 9 blocks, the ragged last one first, in between or last; any -1 between."""
    torch = _torch()
    b, lens = _batch([(32, 39, 5)])     # 1253 tokens: 10 query blocks, 20 key blocks, the last of 37 keys
    heads = 2
    q, k, v = _qkv(14, sum(lens), heads, d, dtype, gain=gain)
    rng = np.random.default_rng(15)
    blocks = np.full((heads, 10, 11), -1, np.int32)
    for h in range(heads):
        for i in range(10):
            pick = rng.permutation(19)[:i]
            if i:
                pick[rng.integers(i)] = 19
            if h == 0:
                blocks[h, i, :i] = np.sort(pick)                 # ascending, as the selection writes them
            else:
                blocks[h, i, rng.permutation(11)[:i]] = pick
    o = _run(b, heads, d, dtype, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda())
    _check(o, q, k, v, blocks, lens, dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_infinite_scores_in_long_lists(dtype, d):
    """As test_infinite_scores, with the keys of -inf in the first half of a list, in the second, in both."""
    torch = _torch()
    b, lens = _batch([(16, 64, 0)])
    q, k, v = _qkv(16, 1024, 1, d, dtype)
    q[:, 0, 0] = q[:, 0, 0].abs() + 0.5
    k[0:512, 0, 0] = -float("inf")      # blocks 0 .. 7
    blocks = np.array([[list(range(16)), list(range(8)) + [-1] * 8, [15 - i for i in range(16)], [7, 9] + [-1] * 14,
                        list(range(8)) + [12] + [-1] * 7, [3] + [-1] * 15, [12] * 8 + [5] * 8, [15] * 16]], np.int32)
    o = _run(b, 1, d, dtype, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda()).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        ref, mag = B.sparse_attention(*(x.double().numpy() for x in (q, k, v)), blocks, mag=True)
    nan = np.r_[128:256, 640:768]
    assert np.isnan(o[nan]).all() and np.isnan(ref[nan]).all()
    keep = np.setdiff1d(np.arange(1024), nan)
    assert (np.abs(o[keep] - ref[keep]) <= (4 * 2.0 ** -8 if dtype == "bf16" else 1e-4) * mag[keep]).all()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_all_blocks_listed_is_dense_attention(dtype, d):
    torch = _torch()
    b, lens = _batch([(20, 20, 39), (1, 1, 0), (12, 13, 5)])
    heads = 2
    q, k, v = _qkv(6, sum(lens), heads, d, dtype)
    n = max(-(-L // 64) for L in lens)
    blocks = np.broadcast_to(np.arange(n, dtype=np.int32), (heads, dit.attention_query_blocks(b), n)).copy()
    o = _run(b, heads, d, dtype, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda())
    _check(o, q, k, v, blocks, lens, dtype)
    nb = dit.attention_workspace_size(b, heads, d, _dt(dtype)[1])
    ws, dense = torch.empty(nb, dtype=torch.uint8, device="cuda"), torch.empty_like(o)
    dit.dit_attention(b, heads, d, _dt(dtype)[1], q.cuda(), k.cuda(), v.cuda(), dense, ws, nb)
    diff = (dense.double() - o.double()).norm() / o.double().norm()
    assert diff < (2.0 ** -7 if dtype == "bf16" else 1e-5)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_unlisted_blocks_and_other_requests_are_not_read(dtype, d):
    """NaN in every unlisted block, in the neighbouring request and behind the last token: the outputs stay finite and right."""
    torch = _torch()
    b, lens = _batch([(10, 10, 0), (13, 13, 20)])   # 100 and 189 tokens: last blocks of 36 and 61 keys
    heads = 2
    q, k, v = _qkv(8, sum(lens), heads, d, dtype)
    blocks = np.full((heads, 3, 2), -1, np.int32)
    blocks[:, 0] = [1, 1]
    blocks[:, 1], blocks[:, 2] = [2, 0], [2, 0]
    kk, vv = k.clone(), v.clone()
    for x in (kk, vv):
        x[:64] = float("nan")
        x[100 + 64:100 + 128] = float("nan")
    pad = torch.full((70, heads, d), float("nan"), dtype=k.dtype)
    dev = [torch.cat([x, pad]).cuda() for x in (kk, vv)]
    o = _run(b, heads, d, dtype, q.cuda(), dev[0], dev[1], torch.from_numpy(blocks).cuda())
    _check(o, q, k, v, blocks, lens, dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_infinite_scores(dtype, d):
    """Keys whose scores are -inf add nothing wherever they lie; a query that sees nothing else is NaN, as in the
    dense attention, and so is one that sees +inf."""
    torch = _torch()
    b, lens = _batch([(16, 20, 0)])
    q, k, v = _qkv(9, 320, 1, d, dtype)
    q[:, 0, 0] = q[:, 0, 0].abs() + 0.5
    k[0:128, 0, 0] = -float("inf")      # blocks 0, 1
    k[256 + 7, 0, 0] = -float("inf")
    blocks = np.array([[[0, 1, 3, 4], [0, 1, -1, -1], [4, 0, 2, 1]]], np.int32)
    o = _run(b, 1, d, dtype, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda()).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        ref, mag = B.sparse_attention(*(x.double().numpy() for x in (q, k, v)), blocks, mag=True)
    assert np.isnan(o[128:256]).all() and np.isnan(ref[128:256]).all()
    keep = np.r_[0:128, 256:320]
    assert (np.abs(o[keep] - ref[keep]) <= (4 * 2.0 ** -8 if dtype == "bf16" else 1e-4) * mag[keep]).all()
    k[200, 0, 0] = float("inf")         # block 3
    o = _run(b, 1, d, dtype, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda())
    assert torch.isnan(o[:128]).all() and torch.isfinite(o[256:]).all()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_sparse_bits_do_not_depend_on_the_batch(dtype, d):
    torch = _torch()
    b, lens = _batch([(9, 9, 50), (24, 24, 11), (2, 2, 0)])
    heads, keep = 2, 4
    q, k, v = (x.cuda() for x in _qkv(10, sum(lens), heads, d, dtype))
    blocks = torch.from_numpy(_lists(11, lens, heads, keep)).cuda()
    packed = _run(b, heads, d, dtype, q, k, v, blocks)
    off = row = 0
    for r, L in zip([(9, 9, 50), (24, 24, 11), (2, 2, 0)], lens):
        nq = -(-L // 128)
        alone = _run(_batch([r])[0], heads, d, dtype, *(x[off:off + L].contiguous() for x in (q, k, v)),
                     blocks[:, row:row + nq].contiguous())
        assert torch.equal(alone, packed[off:off + L])
        off += L
        row += nq


@pytest.mark.parametrize("keep", [5, 10])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_sparse_bits_do_not_depend_on_the_other_queries(dtype, d, keep):
    """One query of a block with scores that grow from key block to key block, so that its maximum rises again and again:
    the bits of every other query of the request stay."""
    torch = _torch()
    b, lens = _batch([(16, 40, 0)])     # 640 tokens: 5 query blocks, 10 key blocks
    heads = 2
    q, k, v = _qkv(22, 640, heads, d, dtype)
    k[:, :, 0] = torch.linspace(-1, 1, 640)[:, None].to(k.dtype) * 4   # what the changed query sees
    q[:, :, 0] = 0
    blocks = np.broadcast_to(np.arange(keep, dtype=np.int32), (heads, 5, keep)).copy()
    dev = [x.cuda() for x in (q, k, v)] + [torch.from_numpy(blocks).cuda()]
    base = _run(b, heads, d, dtype, *dev).clone()
    _check(base, q, k, v, blocks, lens, dtype)
    for at in (0, 3, 37, 100, 300):
        q2 = q.clone()
        q2[at, :, 0] = 40.0
        o = _run(b, heads, d, dtype, q2.cuda(), *dev[1:])
        _check(o, q2, k, v, blocks, lens, dtype)
        same = [i for i in range(640) if i != at]
        assert torch.equal(o[same], base[same]), at


@pytest.mark.parametrize("dtype,d", TYPES)
def test_sparse_bits_do_not_depend_on_the_batch_past_256_query_blocks(dtype, d):
    """Long lists, every call with more query blocks (times heads) than those whose lists are halved."""
    torch = _torch()
    reqs = [(16, 40, 3), (20, 34, 0)]
    b, lens = _batch(reqs)
    heads, keep = 64, 11
    q, k, v = (x.cuda() for x in _qkv(23, sum(lens), heads, d, dtype))
    blocks = torch.from_numpy(_lists(24, lens, heads, keep)).cuda()
    packed = _run(b, heads, d, dtype, q, k, v, blocks)
    off = row = 0
    for r, L in zip(reqs, lens):
        nq = -(-L // 128)
        assert nq * heads > 256
        alone = _run(_batch([r])[0], heads, d, dtype, *(x[off:off + L].contiguous() for x in (q, k, v)),
                     blocks[:, row:row + nq].contiguous())
        assert torch.equal(alone, packed[off:off + L])
        off += L
        row += nq


@pytest.mark.parametrize("keep", [3, 10])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_sparse_output_over_the_queries(dtype, d, keep):
    """o may be q itself."""
    torch = _torch()
    b, lens = _batch([(20, 33, 7), (1, 5, 0)])
    q, k, v = (x.cuda() for x in _qkv(25, sum(lens), 3, d, dtype))
    blocks = torch.from_numpy(_lists(26, lens, 3, keep)).cuda()
    want = _run(b, 3, d, dtype, q, k, v, blocks)
    dit.dit_attention_sparse(b, 3, d, _dt(dtype)[1], q, k, v, blocks, keep, q, None, 0)
    torch.cuda.synchronize()
    assert torch.equal(q, want)


# ---------------------------------------------------------------------------- selection
def _select(b, heads, d, dtype, q, k, keep, flags=0):
    torch = _torch()
    n = dit.attention_select_workspace_size(b, heads, d, _dt(dtype)[1])
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    nq = dit.attention_query_blocks(b)
    out = torch.full((heads * nq * keep + 5,), 123456, dtype=torch.int32, device="cuda")
    dit.dit_attention_select(b, heads, d, _dt(dtype)[1], q, k, keep, flags, out, ws, n)
    torch.cuda.synchronize()
    assert (out[heads * nq * keep:] == 123456).all()
    return out[:heads * nq * keep].view(heads, nq, keep).cpu().numpy()


def _ref_select(q, k, lens, texts, keep):
    out, off = [], 0
    for L, t in zip(lens, texts):
        qq, kk = (x[off:off + L].double().numpy() for x in (q, k))
        out.append(B.select_blocks(qq, kk, keep, t))
        off += L
    return np.concatenate(out, 1)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("text", [0, 1])
@pytest.mark.parametrize("reqs,keep", BATCHES + [([(1, 128, 0), (60, 70, 90)], 17), ([(80, 100, 130)], 1), ([(80, 100, 130)], 128)])
def test_select(reqs, keep, text, dtype, d):
    b, lens = _batch(reqs)
    heads = 2
    q, k, _ = _qkv(sum(lens) + keep, sum(lens), heads, d, dtype)
    got = _select(b, heads, d, dtype, q.cuda(), k.cuda(), keep, dit.DIT_SELECT_TEXT if text else 0)
    assert np.array_equal(got, _ref_select(q, k, lens, [r[2] if text else 0 for r in reqs], keep))


@pytest.mark.parametrize("reqs,heads,keep,text,dtype,d", [
    ([(80, 100, 130)], 64, 32, 1, "bf16", 64),                          # 128 key blocks, many rows
    ([(140, 145, 20)], 1, 50, 1, "f32", 64), ([(140, 145, 20)], 12, 33, 0, "bf16", 64),      # 318, few rows and many
    ([(150, 150, 7)], 1, 40, 0, "bf16", 128), ([(190, 194, 4)], 2, 576, 1, "bf16", 64), ([(190, 194, 4), (9, 9, 0)], 2, 100, 0, "bf16", 128),
    ([(200, 200, 0), (12, 12, 70)], 1, 3, 1, "bf16", 128), ([(256, 256, 4096)], 1, 103, 1, "bf16", 64),
    ([(256, 256, 4097)], 1, 103, 0, "f32", 64),                         # 1089
])
def test_select_at_every_length(reqs, heads, keep, text, dtype, d):
    """Requests at and around the most key blocks that each of the selection's kernels takes."""
    torch = _torch()
    b, lens = _batch(reqs)
    gen = torch.Generator().manual_seed(sum(lens) + heads)
    q, k = (torch.randn((sum(lens), heads, d), generator=gen).to(_dt(dtype)[0]) for _ in range(2))
    got = _select(b, heads, d, dtype, q.cuda(), k.cuda(), keep, dit.DIT_SELECT_TEXT if text else 0)
    assert np.array_equal(got, _ref_select(q, k, lens, [r[2] if text else 0 for r in reqs], keep))


@pytest.mark.parametrize("dtype,d", TYPES)
def test_select_ties_zeros_and_non_finite_scores(dtype, d):
    """Equal scores go to the lower index (all of them, repeated key blocks, both zeros); NaN first; infinities in order."""
    torch = _torch()
    b, lens = _batch([(40, 40, 0)])     # 25 key blocks, 13 query blocks
    q, k, _ = _qkv(12, 1600, 1, d, dtype)
    z = torch.zeros_like(q)
    for keep in (1, 7, 24, 25, 30):
        want = list(range(min(keep, 25))) + [-1] * max(0, keep - 25)
        assert (_select(b, 1, d, dtype, z.cuda(), k.cuda(), keep) == want).all()
        assert (_select(b, 1, d, dtype, (-z).cuda(), z.cuda(), keep) == want).all()
    k[64 * 5:64 * 20] = k[:64].repeat(15, 1, 1)   # blocks 0 and 5 .. 19 alike
    for keep in (3, 9, 16, 20):
        assert np.array_equal(_select(b, 1, d, dtype, q.cuda(), k.cuda(), keep), _ref_select(q, k, lens, [0], keep))
    q = q.abs()
    k[64 * 3 + 5, 0, 2] = float("nan")
    k[64 * 22, 0, 0] = float("inf")
    k[64 * 23, 0, 0] = -float("inf")
    k[64 * 24, 0, 1] = float("inf")
    with np.errstate(invalid="ignore"):
        for keep in (1, 2, 3, 4, 24):
            assert np.array_equal(_select(b, 1, d, dtype, q.cuda(), k.cuda(), keep), _ref_select(q, k, lens, [0], keep))


@pytest.mark.parametrize("dtype,d", TYPES)
def test_select_text_with_nan_and_equal_scores(dtype, d):
    """NaN and infinite scores inside and behind the text's blocks, lists no longer than the text, and scores that
    differ in their last bits only."""
    b, lens = _batch([(30, 30, 130)])   # 1030 tokens: 17 key blocks, 3 of them text
    q, k, _ = _qkv(13, 1030, 2, d, dtype)
    q = q.abs()
    k[5, 0, 0] = k[64 * 9, 0, 3] = float("nan")
    k[64 * 4, 1, 0] = float("inf")
    k[70, 1, 0] = -float("inf")
    with np.errstate(invalid="ignore"):
        for keep in (1, 2, 3, 4, 5, 9, 16, 17, 20):
            for t in (0, 130):
                got = _select(b, 2, d, dtype, q.cuda(), k.cuda(), keep, dit.DIT_SELECT_TEXT if t else 0)
                assert np.array_equal(got, _ref_select(q, k, lens, [t], keep)), (keep, t)
    # scores 1 + j 2^-40: equal high words, told apart by the low ones alone
    q = q * 0
    q[:, :, 0], q[:, :, 1] = 1.0, 2.0 ** -20
    k = k.nan_to_num(0.0, 0.0, 0.0) * 0
    k[:, :, 0] = 1.0
    order = np.random.default_rng(3).permutation(17)
    for j in range(17):
        k[j * 64:(j + 1) * 64, :, 1] = float(order[j] % 12) * 2.0 ** -20
    for keep in (1, 5, 11, 16):
        assert np.array_equal(_select(b, 2, d, dtype, q.cuda(), k.cuda(), keep), _ref_select(q, k, lens, [0], keep)), keep


def test_select_and_attend_at_the_largest_request():
    """2048 key blocks, the most a request may hold: the last block chosen and read."""
    torch = _torch()
    b, lens = _batch([(256, 256, 65536)])
    T = lens[0]
    q, k, v = (torch.zeros((T, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    q[:, 0, 0] = 1
    k[T - 64:, 0, 0] = 1
    k[64 * 1000:64 * 1001, 0, 0] = 2
    v[:, 0, 0] = torch.arange(T, device="cuda").div(64, rounding_mode="floor").remainder(256).to(torch.bfloat16)
    blocks = _select(b, 1, 64, "bf16", q, k, 3)
    assert (blocks == [0, 1000, 2047]).all()
    o = _run(b, 1, 64, "bf16", q, k, v, torch.from_numpy(blocks).cuda())
    p = np.exp(np.array([0.0, 2.0, 1.0]) / 8)
    want = (p * np.array([0, 1000 % 256, 2047 % 256])).sum() / p.sum()
    # three distinct probabilities of 64 equal keys each: bounds as above, sum p |v| = want
    assert (o[:, 0, 0].double() - want).abs().max() <= (3 * 2.0 ** -8 + 1e-4) * want
    assert not o[:, 0, 1:].any()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_sixteen_requests_and_lists_longer_than_any(dtype, d):
    """The most requests a batch may hold, of 1 to 400 tokens, with lists of 2048 entries."""
    torch = _torch()
    reqs = [(1, 1 + r, (r * 37) % 200) for r in range(14)] + [(1, 1, 0), (20, 20, 0)]
    b, lens = _batch(reqs)
    q, k, v = _qkv(17, sum(lens), 2, d, dtype)
    got = _select(b, 2, d, dtype, q.cuda(), k.cuda(), 2048, dit.DIT_SELECT_TEXT)
    assert np.array_equal(got, _ref_select(q, k, lens, [r[2] for r in reqs], 2048))
    blocks = _lists(18, lens, 2, 2048)
    o = _run(b, 2, d, dtype, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda())
    _check(o, q, k, v, blocks, lens, dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_most_heads(dtype, d):
    """65535 heads of 2 tokens: every head's list and output."""
    torch = _torch()
    heads, b = 65535, _batch([(1, 2, 0)])[0]
    gen = torch.Generator(device="cuda").manual_seed(19)
    q, k, v = (torch.randn((2, heads, d), generator=gen, device="cuda").to(_dt(dtype)[0]) for _ in range(3))
    blocks = _select(b, heads, d, dtype, q, k, 2)
    assert (blocks == [0, -1]).all()
    o = _run(b, heads, d, dtype, q, k, v, torch.from_numpy(blocks).cuda()).double()
    q, k, v = (x.double() for x in (q, k, v))
    p = torch.stack([(q * k[j]).sum(2) for j in range(2)], 2) / d ** 0.5   # [query, head, key]
    S = max(q.abs().sum(2).max().item() * k.abs().max().item() / d ** 0.5, 1.0)
    p = p.softmax(2)
    ref = sum(p[:, :, j, None] * v[j] for j in range(2))
    mag = sum(p[:, :, j, None] * v[j].abs() for j in range(2))
    rel = 2 * (d + 3) * 2.0 ** -24 * S + 10 * 2.0 ** -24 + (3 * 2.0 ** -8 if dtype == "bf16" else 0)
    assert ((o - ref).abs() <= rel * mag).all()


@pytest.mark.parametrize("dtype,d,heads", [("bf16", 64, 261), ("bf16", 128, 131), ("f32", 64, 131)])
def test_offsets_past_32_bits(dtype, d, heads):
    """The largest request with q, k and v of more than 4 GiB each: the last heads' last query blocks."""
    torch = _torch()
    b, lens = _batch([(256, 256, 65536)])
    T = lens[0]
    gen = torch.Generator(device="cuda").manual_seed(20)
    q, k, v = (torch.randn((T, heads, d), generator=gen, device="cuda", dtype=_dt(dtype)[0]) for _ in range(3))
    assert q.numel() * q.element_size() > 1 << 32
    blocks = torch.full((heads, T // 128, 3), -1, dtype=torch.int32, device="cuda")
    blocks[-3:, -2:] = torch.tensor([2047, 5, 2046], dtype=torch.int32, device="cuda")
    o = _run(b, heads, d, dtype, q, k, v, blocks)
    assert not o[:, :-3].any() and not o[:-256].any()
    pick = np.r_[5 * 64:6 * 64, 2046 * 64:2048 * 64]
    qq = q[-256:, -3:].double().cpu().numpy()
    kk, vv = (x[torch.from_numpy(pick).cuda(), -3:].double().cpu().numpy() for x in (k, v))
    S = max(np.abs(qq[:, h]).sum(1).max() * np.abs(kk[:, h]).max() for h in range(3)) / d ** 0.5
    rel = 2 * (d + 3) * 2.0 ** -24 * S + 200 * 2.0 ** -24 + (3 * 2.0 ** -8 if dtype == "bf16" else 0)
    got = o[-256:, -3:].double().cpu().numpy()
    for h in range(3):
        p = np.exp(qq[:, h] @ kk[:, h].T / d ** 0.5)
        p /= p.sum(1, keepdims=True)
        assert (np.abs(got[:, h] - p @ vv[:, h]) <= rel * (p @ np.abs(vv[:, h]))).all()
    # the selection over the same tensors: the last query blocks of the last heads
    lists = _select(b, heads, d, dtype, q, k, 40)
    km = [k[:, h].double().view(2048, 64, d).mean(1) for h in range(heads - 3, heads)]
    for i, h in enumerate(range(heads - 3, heads)):
        s = (q[-128:, h].double().mean(0) * km[i]).sum(1)
        assert np.array_equal(lists[h, -1], np.sort(s.topk(40).indices.cpu().numpy()))


# ---------------------------------------------------------------------------- together
def _layer(b, T, heads, d, keep, bufs, stream=None):
    """One attention layer in 8 bits, as a program chains the calls: x -> codes -> q, k, v -> lists -> attention -> codes -> y."""
    H, w = heads * d, bufs
    bf = dit.DIT_BF16
    dit.dit_quantize_fp8(T, H, 1, bf, w["x"], w["xq"], w["xs"], stream)
    for n in "qkv":
        dit.dit_linear_fp8(T, H, H, w["xq"], w["xs"], w["w" + n], w["s" + n], w["b" + n], bf, w[n], bf, stream)
    dit.dit_attention_select(b, heads, d, bf, w["q"], w["k"], keep, dit.DIT_SELECT_TEXT, w["blocks"], w["ws"], w["ws"].numel(), stream)
    dit.dit_attention_sparse(b, heads, d, bf, w["q"], w["k"], w["v"], w["blocks"], keep, w["o"], w["ws"], w["ws"].numel(), stream)
    dit.dit_quantize_fp8(T, H, 1, bf, w["o"], w["xq"], w["xs"], stream)
    dit.dit_linear_fp8(T, H, H, w["xq"], w["xs"], w["wo"], w["so"], w["bo"], bf, w["y"], dit.DIT_F32, stream)


@pytest.mark.parametrize("reqs,keep", [([(16, 16, 77)], 4), ([(20, 24, 33), (9, 7, 0), (1, 1, 0)], 3)])
def test_layer_in_8_bits_eager_and_captured(reqs, keep):
    """Each stage against the reference on the stage's own inputs, then the chain on a side stream and in a HIP graph
    replayed with other inputs and eager work in between: the same bits."""
    torch = _torch()
    b, lens = _batch(reqs)
    T, heads, d = sum(lens), 2, 64
    H = heads * d
    n = max(dit.attention_select_workspace_size(b, heads, d, dit.DIT_BF16),
            dit.attention_sparse_workspace_size(b, heads, d, dit.DIT_BF16))
    w = {"ws": torch.empty(n, dtype=torch.uint8, device="cuda")}
    w["x"] = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    nc, ns = dit.fp8_layout(T, H, 1)
    w["xq"], w["xs"] = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")
    for nm in "qkvo":
        wt = torch.from_numpy(synth.normal(20, "w" + nm, (H, H), std=H ** -0.5)).to(torch.bfloat16).cuda()
        nc, ns = dit.fp8_layout(H, H, 128)
        w["w" + nm], w["s" + nm] = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")
        dit.dit_quantize_fp8(H, H, 128, dit.DIT_BF16, wt, w["w" + nm], w["s" + nm])
        w["b" + nm] = torch.from_numpy(synth.normal(20, "b" + nm, (H,), std=0.1)).to(torch.bfloat16).cuda()
        w[nm] = torch.empty((T, heads, d), dtype=torch.bfloat16, device="cuda")
    w["y"] = torch.empty((T, H), dtype=torch.float32, device="cuda")
    w["blocks"] = torch.empty((heads, dit.attention_query_blocks(b), keep), dtype=torch.int32, device="cuda")
    inputs = [torch.from_numpy(synth.normal(21 + i, "x", (T, H))).to(torch.bfloat16).cuda() for i in range(3)]

    def eager(x):
        w["x"].copy_(x)
        _layer(b, T, heads, d, keep, w)
        torch.cuda.synchronize()
        return w["y"].clone()
    want = [eager(x) for x in inputs]
    # stage by stage, on the last input
    xq, xs = B.quantize_fp8(inputs[2].double().cpu().numpy(), 1)
    xv = B.dequantize_fp8(xq, xs, 1, H)
    host = {k: v.cpu().numpy() for k, v in w.items() if v.dtype in (torch.uint8, torch.int32)}
    for nm in "qkv":
        wv = B.dequantize_fp8(host["w" + nm].reshape(H, -1), host["s" + nm].reshape(1, -1), 128, H)
        ref = xv @ wv.T + w["b" + nm].double().cpu().numpy()
        got = w[nm].double().cpu().numpy().reshape(T, H)
        assert np.linalg.norm(got - ref) / np.linalg.norm(ref) < 2.0 ** -8
    q, k, v, o = (w[nm].cpu() for nm in "qkvo")
    assert np.array_equal(host["blocks"], _ref_select(q, k, lens, [r[2] for r in reqs], keep))
    _check(w["o"], q, k, v, host["blocks"], lens, "bf16")
    oq, os_ = B.quantize_fp8(o.double().numpy().reshape(T, H), 1)
    wv = B.dequantize_fp8(host["wo"].reshape(H, -1), host["so"].reshape(1, -1), 128, H)
    ref = B.dequantize_fp8(oq, os_, 1, H) @ wv.T + w["bo"].double().cpu().numpy()
    assert np.linalg.norm(want[2].double().cpu().numpy() - ref) / np.linalg.norm(ref) < 1e-5
    # a side stream, by handle
    side = torch.cuda.Stream()
    w["x"].copy_(inputs[0])
    side.wait_stream(torch.cuda.current_stream())
    _layer(b, T, heads, d, keep, w, side)
    torch.cuda.synchronize()
    assert torch.equal(w["y"], want[0])
    # captured and replayed
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _layer(b, T, heads, d, keep, w, torch.cuda.current_stream())
    for i in (1, 0, 2, 1):
        w["x"].copy_(inputs[i])
        w["ws"].fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(w["y"], want[i])
        assert torch.equal(eager(inputs[(i + 1) % 3]), want[(i + 1) % 3])


def test_two_layers_at_once():
    """Two chains in flight on two streams, each with buffers of its own, give the bits that each gives alone."""
    torch = _torch()
    heads, d, keep = 4, 64, 6
    b, lens = _batch([(24, 24, 30), (9, 9, 0)])
    T, H = sum(lens), heads * d
    n = dit.attention_select_workspace_size(b, heads, d, dit.DIT_BF16)
    sets = []
    for seed in (30, 31):
        w = {"ws": torch.empty(n, dtype=torch.uint8, device="cuda")}
        w["x"] = torch.from_numpy(synth.normal(seed, "x", (T, H))).to(torch.bfloat16).cuda()
        nc, ns = dit.fp8_layout(T, H, 1)
        w["xq"], w["xs"] = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")
        for nm in "qkvo":
            wt = torch.from_numpy(synth.normal(seed, "w" + nm, (H, H), std=H ** -0.5)).to(torch.bfloat16).cuda()
            nc, ns = dit.fp8_layout(H, H, 128)
            w["w" + nm], w["s" + nm] = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")
            dit.dit_quantize_fp8(H, H, 128, dit.DIT_BF16, wt, w["w" + nm], w["s" + nm])
            w["b" + nm] = torch.from_numpy(synth.normal(seed, "b" + nm, (H,))).to(torch.bfloat16).cuda()
        for nm in "qkv":
            w[nm] = torch.empty((T, heads, d), dtype=torch.bfloat16, device="cuda")
        w["o"] = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
        w["y"] = torch.empty((T, H), dtype=torch.float32, device="cuda")
        w["blocks"] = torch.empty((heads, dit.attention_query_blocks(b), keep), dtype=torch.int32, device="cuda")
        sets.append(w)
    alone = []
    for w in sets:
        _layer(b, T, heads, d, keep, w)
        torch.cuda.synchronize()
        alone.append({k: w[k].clone() for k in ("blocks", "o", "y")})
        assert torch.isfinite(w["y"]).all()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for w in sets:
            for k in ("blocks", "o", "y"):
                w[k].zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for w, s in zip(sets, streams):
                _layer(b, T, heads, d, keep, w, s)
        torch.cuda.synchronize()
        for w, ref in zip(sets, alone):
            assert all(torch.equal(w[k], ref[k]) for k in ref)


def test_calls_without_a_stream_run_on_the_current_one():
    torch = _torch()
    assert dit._stream(None) == torch.cuda.current_stream().cuda_stream
    side = torch.cuda.Stream()
    x = torch.randn((5000, 4096), device="cuda", dtype=torch.bfloat16)
    nc, ns = dit.fp8_layout(5000, 4096, 1)
    q, s = torch.zeros(nc, dtype=torch.uint8, device="cuda"), torch.zeros(ns, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        assert dit._stream(None) == side.cuda_stream == torch.cuda.current_stream().cuda_stream
        for _ in range(20):        # each call waits for the copy ahead of it on the same stream alone
            x.normal_()
            dit.dit_quantize_fp8(5000, 4096, 1, dit.DIT_BF16, x, q, s)
        side.synchronize()
    got = q.clone(), s.clone()
    dit.dit_quantize_fp8(5000, 4096, 1, dit.DIT_BF16, x, q, s)
    torch.cuda.synchronize()
    assert torch.equal(got[0], q) and torch.equal(got[1], s)
