"""Attention of packed sequences with grouped heads on the GPU against 64 bits.

Tolerances.  A score is off by ds = scale (d + 8) 2^-24 |q| |k| (d additions, the products' scaling and the exponent's
argument), which moves its probability by that share.  bf16: each probability is rounded by 2^-8 of it, in the sum that
divides as in the one that is divided; fp32: a step 2^-24 for each of the keys' additions in either sum, and as many for
the maxima's rescaling.  All that of the sum of p |v|, and the output's own half step (2^-8 or 2^-24)."""
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


def _reference(q, k, v, ql, kl, rows, scale, causal):
    """o, sum of p |v| and the largest |q| |k|, in 64 bits on the GPU; keys past what a query sees are cut off, not multiplied by 0."""
    torch = _torch()
    G = q.shape[1] // k.shape[1]
    o = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    mag = torch.zeros_like(o)
    at, top = 0, 0.0
    for n, m, f in zip(ql, kl, rows):
        if n and m:
            qn = q[at:at + n].double().norm(dim=2).nan_to_num(0, 0).max()
            kn = k[f:f + m].double().norm(dim=2).nan_to_num(0, 0).max()
            top = max(top, float(qn * kn))
        for h in range(q.shape[1]):
            kh, vh = k[f:f + m, h // G].double(), v[f:f + m, h // G].double()
            clean = bool(torch.isfinite(kh).all() and torch.isfinite(vh).all())
            for i in range(0, n, n if clean and n else 1):
                r = n if clean else i + 1
                most = max(0, min(m, m - n + r)) if causal else m
                if most == 0:
                    continue
                s = scale * (q[at + i:at + r, h].double() @ kh[:most].t().contiguous())
                if causal and r - i > 1:
                    lim = torch.arange(m - n + i, m - n + r, device=q.device)[:, None]
                    s = s.masked_fill(torch.arange(most, device=q.device)[None] > lim, -math.inf)
                p = torch.softmax(s, 1)
                if causal and r - i > 1:
                    p = p.nan_to_num(0.0)  # rows that see nothing
                o[at + i:at + r, h] = p @ vh[:most]
                mag[at + i:at + r, h] = p @ vh[:most].abs()
        at += n
    return o, mag, top


def _check(got, ref, mag, top, keys, d, scale, dtype):
    torch = _torch()
    ds = abs(scale) * (d + 8) * 2.0 ** -24 * top
    if dtype == "bf16":
        tol = (2 * 2.0 ** -8 + 4 * ds) * mag + 2.0 ** -8 * ref.abs()
    else:
        tol = ((4 * keys + 64) * 2.0 ** -24 + 4 * ds) * mag + 2.0 ** -24 * ref.abs()
    got = got.double()
    assert bool(torch.equal(torch.isnan(got), torch.isnan(ref)))
    ok = torch.isfinite(ref)
    assert bool(torch.equal(torch.isfinite(got), ok))
    off = (got - ref).abs()[ok] - tol[ok]
    assert off.numel() == 0 or float(off.max()) <= 0, float(((got - ref).abs()[ok] / tol[ok].clamp(min=1e-300)).max())


class Case:
    """Inputs of a call: fused rows [q | k | v], or a cache in slots; o between guard rows."""

    def __init__(self, ql, kl, heads, kv_heads, d, dtype, cache=False, seed=0, std=1.0, rows=None, gap=0):
        torch = _torch()
        self.ql, self.kl, self.heads, self.kv_heads, self.d, self.dtype = list(ql), list(kl), heads, kv_heads, d, dtype
        dt = _dt(dtype)[0]
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: (std * torch.randn(s, generator=gen, device="cuda")).to(dt)
        self.rows, at = [], 0
        for m in self.kl:
            self.rows.append(at)
            at += m + (70 if cache else 0)
        if rows is not None:
            self.rows = list(rows)
        total, nq = max(at, 1), max(sum(self.ql), 1)
        if cache or self.ql != self.kl:
            self.q = rnd(nq, heads, d)
            kv = torch.full((total, 2 * kv_heads + gap, d), math.nan, dtype=dt, device="cuda")
            for f, m in zip(self.rows, self.kl):
                kv[f:f + m] = rnd(m, 2 * kv_heads + gap, d)
            self.k, self.v = kv[:, :kv_heads], kv[:, kv_heads:2 * kv_heads]
        else:
            x = rnd(total, heads + 2 * kv_heads + gap, d)
            self.q, self.k, self.v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:heads + 2 * kv_heads]
        self.packed = rows is None and not cache

    def run(self, causal, scale=None, o=None, ws=None):
        torch = _torch()
        code = _dt(self.dtype)[1]
        scale = 1 / math.sqrt(self.d) if scale is None else scale
        seqs = dit.Sequences(self.ql, self.kl, None if self.packed else self.rows)
        n = dit.attention_grouped_workspace_size(seqs, self.heads, self.kv_heads, self.d, code)
        if ws is None:
            ws = torch.full((n + 512,), 0xff, dtype=torch.uint8, device="cuda")  # NaN in every type
            end = ws[n:].clone()
        else:
            end = None
        guard = None
        if o is None:
            guard = torch.full((sum(self.ql) + 2, self.heads, self.d), 3.0, dtype=self.q.dtype, device="cuda")
            o = guard[1:-1]
        dit.dit_attention_grouped(seqs, self.heads, self.kv_heads, self.d, code, dit.DIT_CAUSAL if causal else 0, scale, self.q,
                                  self.q.stride(0), self.k, self.v, self.k.stride(0), o if o.numel() else guard, o.stride(0), ws, n)
        torch.cuda.synchronize()
        assert guard is None or ((guard[0] == 3).all() and (guard[-1] == 3).all())
        assert end is None or torch.equal(ws[n:], end)
        return o

    def verify(self, causal, scale=None):
        o = self.run(causal, scale)
        scale = 1 / math.sqrt(self.d) if scale is None else scale
        nq = sum(self.ql)
        ref, mag, top = _reference(self.q[:nq], self.k, self.v, self.ql, self.kl, self.rows, scale, causal)
        _check(o, ref, mag, top, max(self.kl), self.d, scale, self.dtype)
        return o


TYPES = [("bf16", 64), ("bf16", 128), ("f32", 64)]
HEADS = [(1, 1), (6, 3), (5, 5), (8, 1), (24, 8), (40, 8)]
PROMPTS = [[1], [2, 1, 3], [63], [64], [65, 1], [128, 127, 129], [300, 5, 64, 191], [1, 1, 1, 1, 1], [577], [1025, 33]]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("lens", PROMPTS, ids=str)
def test_prompts(lens, dtype, d, causal):
    heads, kv = HEADS[sum(lens) % len(HEADS)]
    Case(lens, lens, heads, kv, d, dtype, seed=sum(lens)).verify(causal)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("heads,kv", HEADS + [(12, 4), (16, 2), (33, 1), (7, 7)])
def test_head_groups(heads, kv, dtype, d):
    Case([70, 3, 200], [70, 3, 200], heads, kv, d, dtype, seed=heads, gap=1).verify(True)
    Case([1, 3, 20], [70, 333, 64], heads, kv, d, dtype, cache=True, seed=heads).verify(True)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("kl", [[1], [2, 63, 64, 65], [500, 1, 77, 3000], [4097], [9000, 31], [127] * 30], ids=lambda v: str(v[:4]))
@pytest.mark.parametrize("heads,kv", [(32, 8), (6, 6), (16, 1)])
def test_one_token_over_a_cache(kl, heads, kv, dtype, d):
    c = Case([1] * len(kl), kl, heads, kv, d, dtype, cache=True, seed=kl[0])
    a = c.verify(True)
    b = c.run(False)
    assert _torch().equal(a, b)  # a single token sees everything either way


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("ql,kl", [([5, 64, 1, 130], [100, 64, 900, 2000]), ([0, 3, 0], [50, 0, 0]), ([10], [4]), ([200, 3], [70, 1]),
                                   ([33, 0, 7], [5000, 10, 7]), ([600], [4000]), ([200, 1, 3, 40, 1], [9000, 5000, 100, 70, 2049])], ids=str)
def test_parts_of_prompts_and_empty_rows(ql, kl, dtype, d, causal):
    """Queries that continue a cache, sequences without queries or keys, queries ahead of the first key."""
    c = Case(ql, kl, 6, 3, d, dtype, cache=True, seed=sum(kl))
    o = c.verify(causal)
    at = 0
    for n, m in zip(ql, kl):
        none = n if m == 0 else max(0, n - m) if causal else 0
        assert (o[at:at + none] == 0).all()
        at += n


@pytest.mark.parametrize("dtype,d", TYPES)
def test_nothing_to_do(dtype, d):
    """Only sequences without queries: nothing is written (Case.run's guards)."""
    Case([0, 0], [10, 0], 6, 3, d, dtype, cache=True).run(True)
    Case([0], [3000], 6, 3, d, dtype, cache=True).run(False)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_rows_shared_by_sequences(dtype, d):
    """Sequences that read the same rows, or overlapping ones."""
    Case([2, 2, 5], [100, 90, 40], 6, 3, d, dtype, cache=True, rows=[0, 0, 60]).verify(True)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("std", [4.0, 12.0])
def test_large_scores(dtype, d, std):
    """Scores up to thousands: the running max rises often and late."""
    Case([257, 40], [257, 40], 6, 3, d, dtype, std=std, seed=3).verify(True)
    Case([1, 2], [2000, 700], 6, 3, d, dtype, cache=True, std=std, seed=4).verify(True)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0, 2.0 ** -64, 2.0 ** -65])
def test_scales(scale, dtype, d):
    c = Case([130, 5], [130, 5], 6, 3, d, dtype, seed=5)
    if scale >= 2.0 ** -64:
        c.verify(True, scale)
    else:
        with pytest.raises(dit.DitError):
            c.run(True, scale)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("what", ["k", "v", "kv"])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_what_a_query_does_not_see_does_not_reach_it(dtype, d, what, bad):
    """A key or a value that is not finite: queries before it are as if it were not there, those after it take part in it."""
    torch = _torch()
    for lens, at in (([150, 40], 100), ([70], 69), ([300], 64), ([300], 191)):
        clean = Case(lens, lens, 6, 3, d, dtype, seed=6)
        want = clean.run(True).clone()
        c = Case(lens, lens, 6, 3, d, dtype, seed=6)
        if "k" in what:
            c.k[at, 1, 5] = bad
        if "v" in what:
            c.v[at, 1, 7] = bad
        got = c.run(True)
        assert bool(torch.equal(got[:at], want[:at]))
        others = [h for h in range(6) if h // 2 != 1]
        assert bool(torch.equal(got[:, others], want[:, others]) and torch.equal(got[lens[0]:], want[lens[0]:]))
        if "v" in what:
            hit = got[at:lens[0], 2:4, 7]
            assert not torch.isfinite(hit).any()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_infinite_scores(dtype, d):
    """Keys whose scores are -inf for every query of a tile, and a row of which all are."""
    torch = _torch()
    c = Case([200], [200], 2, 1, d, dtype, seed=7)
    c.q[:, :, 0] = 1.0
    c.k[:130, :, 0] = -math.inf
    o = c.run(True)
    scale = 1 / math.sqrt(d)
    ref, mag, top = _reference(c.q[130:], c.k[130:], c.v[130:], [70], [70], [0], scale, True)
    _check(o[130:], ref, mag, top, 200, d, scale, dtype)
    assert torch.isnan(o[:130]).all()  # softmax over -inf alone


@pytest.mark.parametrize("dtype,d", TYPES)
def test_in_place_and_repeatable(dtype, d):
    torch = _torch()
    for lens in ([90, 1, 260], [33] * 5):
        c = Case(lens, lens, 6, 3, d, dtype, seed=8)
        a, b = c.run(True).clone(), c.run(True)
        assert bool(torch.equal(a, b))
        k, v = c.k.clone(), c.v.clone()
        c.run(True, o=c.q)
        assert bool(torch.equal(c.q, a) and torch.equal(c.k, k) and torch.equal(c.v, v))
    c = Case([1, 2], [3000, 900], 6, 3, d, dtype, cache=True, seed=9)
    a = c.run(True).clone()
    c.run(True, o=c.q)
    assert bool(torch.equal(c.q, a))


def test_a_cache_past_32_bit_offsets():
    """Rows of K and V past 2^32 bytes and 2^31 elements."""
    torch = _torch()
    rows, kv, d = (1 << 31) // 256 + 5000, 2, 128
    k = torch.empty((rows, kv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty((rows, kv, d), dtype=torch.bfloat16, device="cuda")
    first = [rows - 3000, 10]
    kl, ql = [3000, 100], [5, 1]
    gen = torch.Generator(device="cuda").manual_seed(1)
    for f, m in zip(first, kl):
        k[f:f + m] = torch.randn((m, kv, d), generator=gen, device="cuda").to(torch.bfloat16)
        v[f:f + m] = torch.randn((m, kv, d), generator=gen, device="cuda").to(torch.bfloat16)
    c = Case([5, 1], [3000, 100], 8, kv, d, "bf16", cache=True)
    c.k, c.v, c.rows = k, v, first
    c.verify(True)


def test_many_sequences():
    lens = [(i * 37) % 90 + 1 for i in range(128)]
    Case(lens, lens, 6, 3, 64, "bf16", seed=2).verify(True)
    Case([1] * 128, [(i * 53) % 400 + 1 for i in range(128)], 8, 2, 128, "bf16", cache=True, seed=2).verify(True)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_two_graphs_with_a_workspace_each(dtype, d):
    """Two captured calls, replayed in turn and with eager calls between, each on its own workspace."""
    torch = _torch()
    cases = [Case([1, 1, 1], [2500, 800, 70], 6, 3, d, dtype, cache=True, seed=1), Case([40, 7], [40, 7], 6, 3, d, dtype, seed=2)]
    graphs, outs, keep = [], [], []
    code = _dt(dtype)[1]
    for c in cases:
        seqs = dit.Sequences(c.ql, c.kl, c.rows)
        n = dit.attention_grouped_workspace_size(seqs, 6, 3, d, code)
        ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
        o = torch.empty((sum(c.ql), 6, d), dtype=c.q.dtype, device="cuda")
        call = lambda c=c, seqs=seqs, ws=ws, o=o, n=n: dit.dit_attention_grouped(
            seqs, 6, 3, d, code, dit.DIT_CAUSAL, 0.1, c.q, c.q.stride(0), c.k, c.v, c.k.stride(0), o, 6 * d, ws, n)
        call()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
        outs.append(o)
        keep.append((ws, call))
    for rep in range(3):
        for c in cases:
            c.q += 0.125
        want = []
        for c, o, (_, call) in zip(cases, outs, keep):
            call()
            torch.cuda.synchronize()
            want.append(o.clone())
            o.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, r in zip(outs, want):
            assert torch.equal(o, r), rep


def _fp4(x):
    torch = _torch()
    rows, K = x.shape
    nc, ns = dit.fp4_layout(rows, K)
    q, s = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")
    dit.dit_quantize_fp4(rows, K, dit.DIT_BF16, x, q, s)
    return q, s


def test_an_encoder_layer_and_one_token_more():
    """Quantise, the fused 4-bit q, k, v product, rotary positions in place, causal attention on the fused rows, the output
    product in 4 bits; then one more token of each prompt over a cache that holds the prompts' keys: the same rows as
    those of the longer prompts."""
    torch = _torch()
    heads, kv, d, H = 8, 2, 64, 512
    lens, more = [37, 130, 1], [38, 131, 2]
    W = heads * d + 2 * kv * d
    gen = torch.Generator(device="cuda").manual_seed(12)
    rnd = lambda std, *s: (std * torch.randn(s, generator=gen, device="cuda")).to(torch.bfloat16)
    wqkv, wo = rnd(H ** -0.5, W, H), rnd(H ** -0.5, H, heads * d)
    bias = rnd(0.1, W)
    x = rnd(1.0, sum(more), H)          # the longer prompts
    starts = [0, 38, 169]
    short = torch.cat([torch.arange(f, f + n) for f, n in zip(starts, lens)]).cuda()
    new = torch.tensor([f + n for f, n in zip(starts, lens)]).cuda()
    w = dit.rope_frequencies(d, 10000.0, 4.0, 64.0, 1.0, 4.0)
    qw, qo = _fp4(wqkv), _fp4(wo)

    def linear(t, wq, N, K, b=None):
        t = t.contiguous()
        q, s = _fp4(t)
        y = torch.empty((t.shape[0], N), dtype=torch.bfloat16, device="cuda")
        dit.dit_linear_fp4(t.shape[0], N, K, q, s, wq[0], wq[1], b, dit.DIT_BF16, y, dit.DIT_BF16)
        return y

    def qkv(t, pos):
        y = linear(t, qw, W, H, bias)
        dit.dit_rope(t.shape[0], heads + kv, d, d, dit.DIT_ROPE_HALF, dit.DIT_BF16, pos.int().contiguous(), w, 1.0, y, W, y, W)
        return y

    def attend(rows, ql, kl, first, k, v, ldkv):
        seqs = dit.Sequences(ql, kl, first)
        n = dit.attention_grouped_workspace_size(seqs, heads, kv, d, dit.DIT_BF16)
        ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
        o = torch.empty((rows.shape[0], heads * d), dtype=torch.bfloat16, device="cuda")
        dit.dit_attention_grouped(seqs, heads, kv, d, dit.DIT_BF16, dit.DIT_CAUSAL, d ** -0.5, rows, W, k, v, ldkv, o, heads * d, ws, n)
        return linear(o, qo, H, heads * d), o

    def prompts(t, ns):
        pos = torch.cat([torch.arange(n) for n in ns]).cuda()
        y = qkv(t, pos)
        out, o = attend(y, ns, ns, None, y[:, heads * d:], y[:, (heads + kv) * d:], W)
        return y, out, o

    y, out, o = prompts(x, more)
    # 64 bits, from the bf16 inputs through the same roundings of the operands
    val = lambda t: T.dequantize_fp4(*T.quantize_fp4(t.double().cpu().numpy()), t.shape[1])
    ref = val(x) @ val(wqkv).T + bias.double().cpu().numpy()
    pos = np.concatenate([np.arange(n) for n in more])
    turned = T.rope(ref.reshape(-1, heads + 2 * kv, d)[:, :heads + kv], pos, list(w), "half")
    got = y.double().cpu().numpy().reshape(-1, heads + 2 * kv, d)
    # two roundings to bf16 on the way (the product's, the turned one's, which mixes two values)
    pair = np.abs(ref.reshape(-1, heads + 2 * kv, d)[:, :heads + kv])
    pair = pair + np.concatenate([pair[:, :, d // 2:], pair[:, :, :d // 2]], 2)
    assert (np.abs(got[:, :heads + kv] - turned) <= 2.0 ** -7 * pair + 1e-4).all()
    assert (np.abs(got[:, heads + kv:] - ref.reshape(-1, heads + 2 * kv, d)[:, heads + kv:]) <= 2.0 ** -8 * np.abs(ref).max()).all()
    gq, gk, gv = got[:, :heads], got[:, heads:heads + kv], got[:, heads + kv:]
    ro, mag = T.grouped_attention(gq, gk, gv, more, more, starts, d ** -0.5, True)
    assert (np.abs(o.double().cpu().numpy().reshape(ro.shape) - ro) <= (2 * 2.0 ** -8 + 1e-4) * mag + 2.0 ** -8 * np.abs(ro)).all()
    rout = val(o) @ val(wo).T
    assert np.linalg.norm(out.double().cpu().numpy() - rout) < 2.0 ** -8 * np.linalg.norm(rout)

    # the prompts without their last token into a cache, then that token
    ys, _, _ = prompts(x[short], lens)
    slot = [5, 300, 100]
    ck, cv = (torch.full((500, kv * d), math.nan, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    at = 0
    for f, n in zip(slot, lens):
        ck[f:f + n], cv[f:f + n] = ys[at:at + n, heads * d:(heads + kv) * d], ys[at:at + n, (heads + kv) * d:]
        at += n
    yt = qkv(x[new], torch.tensor(lens).cuda())
    for i, (f, n) in enumerate(zip(slot, lens)):
        ck[f + n], cv[f + n] = yt[i, heads * d:(heads + kv) * d], yt[i, (heads + kv) * d:]
    _, ot = attend(yt, [1, 1, 1], more, slot, ck, cv, kv * d)
    a, b = ot.double(), o[new].double()
    # either is within the attention's own bound of the same values; the rows they read agree to a rounding
    assert float((a - b).norm() / b.norm()) < 2.0 ** -6


def test_two_layers_at_once_on_two_streams():
    """Quantise, product, rotary positions in place and attention, once after the other, then side by side on streams of
    their own with buffers of their own: the same bits."""
    torch = _torch()
    heads, kv, d, K = 24, 8, 64, 8192
    W = (heads + 2 * kv) * d
    gen = torch.Generator(device="cuda").manual_seed(21)
    rnd = lambda std, *s: (std * torch.randn(s, generator=gen, device="cuda")).to(torch.bfloat16)
    w = dit.rope_frequencies(d, 10000.0)
    wq, ws = _fp4(rnd(K ** -0.5, W, K))

    class Layer:
        def __init__(self, ql, kl):
            self.rows = sum(ql)
            self.x, self.qs = rnd(1.0, self.rows, K), dit.fp4_layout(self.rows, K)
            self.codes, self.scales = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in self.qs)
            self.y = torch.empty((self.rows, W), dtype=torch.bfloat16, device="cuda")
            self.o = torch.empty((self.rows, heads * d), dtype=torch.bfloat16, device="cuda")
            self.seqs = dit.Sequences(ql, kl, None if ql == kl else [0] * len(ql))
            self.cache = None if ql == kl else rnd(1.0, max(kl), 2 * kv * d)
            self.n = dit.attention_grouped_workspace_size(self.seqs, heads, kv, d, dit.DIT_BF16)
            self.ws = torch.empty(max(self.n, 256), dtype=torch.uint8, device="cuda")

        def run(self):
            dit.dit_quantize_fp4(self.rows, K, dit.DIT_BF16, self.x, self.codes, self.scales)
            dit.dit_linear_fp4(self.rows, W, K, self.codes, self.scales, wq, ws, None, dit.DIT_BF16, self.y, dit.DIT_BF16)
            dit.dit_rope(self.rows, heads + kv, d, d, dit.DIT_ROPE_HALF, dit.DIT_BF16, None, w, 1.0, self.y, W, self.y, W)
            k, v, ld = ((self.y[:, heads * d:], self.y[:, (heads + kv) * d:], W) if self.cache is None
                        else (self.cache, self.cache[:, kv * d:], 2 * kv * d))
            dit.dit_attention_grouped(self.seqs, heads, kv, d, dit.DIT_BF16, dit.DIT_CAUSAL, 0.125, self.y, W, k, v, ld, self.o,
                                      heads * d, self.ws, self.n)

    layers = [Layer([4096, 204], [4096, 204]), Layer([1] * 40, [9000] * 20 + [333] * 20), Layer([2000, 1], [2000, 1])]
    want = []
    for layer in layers:
        layer.run()
        want.append(layer.o.clone())
        assert torch.isfinite(layer.o).all()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(3):
        for layer in layers:
            layer.o.zero_()
        torch.cuda.synchronize()
        for layer, s in zip(layers, streams):
            with torch.cuda.stream(s):
                layer.run()
        torch.cuda.synchronize()
        for layer, r in zip(layers, want):
            assert torch.equal(layer.o, r)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_queries_without_any_key(dtype, d, causal):
    """k and v without a row, whose tensors have no address: zeros, for one token as for many."""
    torch = _torch()
    dt, code = _dt(dtype)
    kv = torch.empty((0, 2, 3, d), dtype=dt, device="cuda")
    for ql, kl, first in (([1], [0], None), ([5, 0, 200], [0, 0, 0], None), ([0, 3], [40, 0], [7, 1 << 20])):
        seqs = dit.Sequences(ql, kl, first)
        assert dit.attention_grouped_workspace_size(seqs, 6, 3, d, code) == 0
        q = torch.full((sum(ql), 6, d), math.nan, dtype=dt, device="cuda")
        o = torch.full((sum(ql) + 2, 6, d), 3.0, dtype=dt, device="cuda")
        dit.dit_attention_grouped(seqs, 6, 3, d, code, dit.DIT_CAUSAL if causal else 0, 0.1, q, 6 * d, kv[:, 0], kv[:, 1],
                                  6 * d, o[1:-1], 6 * d, None, 0)
        torch.cuda.synchronize()
        assert (o[0] == 3).all() and (o[-1] == 3).all() and (o[1:-1] == 0).all()
