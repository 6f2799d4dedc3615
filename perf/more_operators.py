"""Timed cases of 4-bit products, rotary positions and grouped attention.

Each case is what a serving program runs on the GPU around a request's text and its products:
  op "quantize"   ``dit_quantize_fp4`` and back: a matrix to e2m1 codes with one power-of-two scale per 1 x 32 block, and the
                  values that these stand for (``dit_dequantize_fp4``)
  op "linear"     ``dit_quantize_fp4`` of the activations and ``dit_linear_fp4`` with weights that are in 4 bits already
  op "rope"       ``dit_rope``: rotary positions of the query and key heads, in either layout, on the whole head or a part of it
  op "attention"  ``dit_attention_grouped``: packed sequences of different lengths, fewer key heads than query heads, causal or not

Sizes are those of the served models (``paper_2510_01565_amd/workloads.py``: text embeddings 4096 wide, 333 or 512 text tokens,
the 1536-wide model with 24 heads of 64, the small fp32 model with 6 heads of 64) and generic powers of two.  With ``own`` false
``run`` computes the same in elementary torch operations.

A case is a dict of plain values: "op", and
  quantize   rows, K, dtype ("bf16" or "f32")
  linear     M, N, K, bias, out ("bf16" or "f32")
  rope       rows, heads, d, rot (dimensions that turn), layout ("half" or "pairs"), dtype, far (largest position), factor (of the
             context's extension, 1: none)
  attention  q, kv ("N,N,..." queries and keys of each sequence), heads, kv_heads, d, dtype, causal, cache (keys in slots of a cache,
             or beside the queries in the rows of one product)
"""
import math

import torch

own = False

BLOCK = 32           # elements of a scale's block
THETA = 500000.0
ORIGINAL = 8192      # positions of the context before its extension
LOW, HIGH = 1.0, 4.0  # turns over it below which a frequency is divided by the factor, above which it is kept


def listed():
    return [
        # four tokens' activations ahead of a product: latency alone
        {"name": "quantize_tokens", "op": "quantize", "rows": 4, "K": 4096, "dtype": "bf16"},
        # the hidden MLP activations of a 2048 px request of the 1536-wide model, an odd row count
        {"name": "quantize_mlp_2048px", "op": "quantize", "rows": 16717, "K": 6144, "dtype": "bf16"},
        # one token through a text encoder's MLP: every weight is read for one row
        {"name": "linear_token", "op": "linear", "M": 1, "N": 16384, "K": 4096, "bias": False, "out": "bf16"},
        # one prompt's output product in a text encoder as wide as the text embeddings
        {"name": "linear_prompt", "op": "linear", "M": 333, "N": 4096, "K": 4096, "bias": False, "out": "bf16"},
        # the first MLP product at 1024 px, kept in 32 bits
        {"name": "linear_1024px_f32", "op": "linear", "M": 4429, "N": 6144, "K": 1536, "bias": True, "out": "f32"},
        # a wide model's MLP product at 2048 px: the largest product
        {"name": "linear_wide_2048px", "op": "linear", "M": 16896, "N": 16384, "K": 4096, "bias": True, "out": "bf16"},
        # sixteen sequences one token further, far past the length that the frequencies were made for
        {"name": "rope_tokens", "op": "rope", "rows": 16, "heads": 40, "d": 128, "rot": 128, "layout": "half", "dtype": "bf16",
         "far": 131071, "factor": 8.0},
        # packed prompts, neighbouring dimensions in pairs, half of each head turned
        {"name": "rope_prompts", "op": "rope", "rows": 16391, "heads": 40, "d": 128, "rot": 64, "layout": "pairs", "dtype": "bf16",
         "far": 16383, "factor": 1.0},
        # the small fp32 model's heads over the text of three requests, two queries' heads to a key head
        {"name": "attention_small_f32", "op": "attention", "q": "32,288,77", "kv": "32,288,77", "heads": 6, "kv_heads": 3, "d": 64,
         "dtype": "f32", "causal": True, "cache": False},
        # the prompts of twelve requests, from one token to four thousand
        {"name": "attention_prompts", "op": "attention", "q": "333,512,77,1,1024,333,2048,130,640,4096,19,256",
         "kv": "333,512,77,1,1024,333,2048,130,640,4096,19,256", "heads": 24, "kv_heads": 8, "d": 64, "dtype": "bf16", "causal": True,
         "cache": False},
        # one token for each of sixteen sequences over their caches
        {"name": "attention_tokens", "op": "attention", "q": "1,1,1,1,1,1,1,1,1,1,1,1,1,1,1,1",
         "kv": "4097,333,16384,1,7000,512,1500,2049,12000,77,900,3500,8192,260,5555,640", "heads": 32, "kv_heads": 8, "d": 128,
         "dtype": "bf16", "causal": True, "cache": True},
        # one long document
        {"name": "attention_long", "op": "attention", "q": "16384", "kv": "16384", "heads": 32, "kv_heads": 8, "d": 128,
         "dtype": "bf16", "causal": True, "cache": False},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choices(["quantize", "linear", "rope", "attention"], [2, 4, 2, 5])[0]
    if op == "quantize":
        rows, K = _log_int(rng, 1, 24000), _log_int(rng, 16, 16384)
        while rows * K > 16717 * 6144:
            rows = rows * 3 // 4
        return {"op": op, "rows": rows, "K": K, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "linear":
        M, N, K = _log_int(rng, 1, 24000), _log_int(rng, 48, 16384), _log_int(rng, 64, 16384)
        if rng.random() < 0.5:
            N, K = -(-N // 64) * 64, -(-K // 64) * 64
        while M * N * K > 16896 * 16384 * 4096:
            M = M * 3 // 4
        return {"op": op, "M": M, "N": N, "K": K, "bias": rng.random() < 0.6, "out": rng.choice(["bf16", "bf16", "f32"])}
    if op == "rope":
        rows, heads, d = _log_int(rng, 1, 20000), _log_int(rng, 1, 64), rng.choice([64, 80, 96, 128, 256])
        while rows * heads * d > 16391 * 40 * 128:
            rows = rows * 3 // 4
        rot = rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)])
        return {"op": op, "rows": rows, "heads": heads, "d": d, "rot": rot, "layout": rng.choice(["half", "pairs"]),
                "dtype": rng.choice(["bf16", "bf16", "f32"]), "far": _log_int(rng, 1, 1000000),
                "factor": rng.choice([1.0, 1.0, 4.0, 8.0, 32.0])}
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = 64 if dtype == "f32" else rng.choice([64, 128, 128])
    heads, kv_heads = rng.choice([(6, 3), (12, 12), (16, 1), (24, 8), (32, 8), (40, 8), (32, 4)])
    kind = rng.choice(["prompts", "prompts", "tokens", "mixed"])
    n = _log_int(rng, 1, 32)
    most = (16384 if dtype == "bf16" else 4096) if kind != "tokens" else 65536
    q, kv = [], []
    for _ in range(n):
        m = _log_int(rng, 1, most)
        c = m if kind == "prompts" else 1 if kind == "tokens" else rng.choice([1, min(m, _log_int(rng, 1, 512)), m])
        q.append(c)
        kv.append(m)
    cost = lambda: sum(a * b for a, b in zip(q, kv)) * heads * d * (6 if dtype == "f32" else 1)
    while (cost() > 16384 * 16384 * 32 * 128 or sum(kv) * kv_heads * d > 131072 * 8 * 128) and len(q) > 1:
        q.pop()
        kv.pop()
    while cost() > 16384 * 16384 * 32 * 128:
        kv[0] = kv[0] * 3 // 4
        q[0] = min(q[0], kv[0])
    return {"op": op, "q": ",".join(map(str, q)), "kv": ",".join(map(str, kv)), "heads": heads, "kv_heads": kv_heads, "d": d,
            "dtype": dtype, "causal": rng.random() < 0.8, "cache": kind != "prompts"}


# ---------------------------------------------------------------------------- shapes and inputs
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _up(a, b):
    return -(-a // b)


def _lengths(case):
    return [int(x) for x in case["q"].split(",")], [int(x) for x in case["kv"].split(",")]


def _slots(case):
    """First row of each sequence's keys and how many rows there are: packed, or slots of a cache with room for 256 more."""
    _, kv = _lengths(case)
    first, at = [], 0
    for n in kv:
        first.append(at)
        at += (_up(n, 256) + 1) * 256 if case["cache"] else n
    return first, at


class _Draws:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)

    def normal(self, shape, std=1.0):
        x = torch.randn(shape, generator=self.gen, device="cuda", dtype=torch.float32)
        return x if std == 1.0 else x.mul_(std)

    def tokens(self, shape):
        """Rows of which neighbours resemble each other."""
        x = self.normal(shape)
        x += 0.7 * self.normal((_up(shape[0], 32),) + shape[1:]).repeat_interleave(32, 0)[: shape[0]]
        return x


def _matrix(dr, rows, K):
    """Normal values whose rows and channels differ in size, as activations' do."""
    x = dr.normal((rows, K))
    x *= torch.exp(0.5 * dr.normal((rows, 1)))
    x *= torch.exp(0.5 * dr.normal((1, K)))
    return x


def _frequencies(case):
    """The frequencies of the rotation in 64 bits, on the host."""
    out = []
    for i in range(case["rot"] // 2):
        w = THETA ** (-2.0 * i / case["rot"])
        g = min(1.0, max(0.0, (ORIGINAL * w / (2 * math.pi) - LOW) / (HIGH - LOW)))
        out.append(w * (g + (1 - g) / case["factor"]))
    return out


def _magnitude(case):
    return 1.0 + 0.1 * math.log(case["factor"])


def _inputs(case, seed):
    dr, op = _Draws(seed), case["op"]
    if op in ("quantize", "linear"):
        rows, K = (case["rows"], case["K"]) if op == "quantize" else (case["M"], case["K"])
        s = {"x": _matrix(dr, rows, K).to(_dtype(case.get("dtype", "bf16")))}
        if op == "linear":
            s["wq"], s["ws"] = _pack(*_quantize(dr.normal((case["N"], K), 0.02).to(torch.bfloat16)))
            s["b"] = dr.normal((case["N"],), 0.02).to(torch.bfloat16) if case["bias"] else None
        return s
    dt = _dtype(case["dtype"])
    if op == "rope":
        x = dr.tokens((case["rows"], case["heads"], case["d"])).to(dt)
        return {"x": x, "pos": torch.randint(0, case["far"] + 1, (case["rows"],), generator=dr.gen, device="cuda", dtype=torch.int32)}
    q, _ = _lengths(case)
    rows, H, Hk, d = _slots(case)[1], case["heads"], case["kv_heads"], case["d"]
    if case["cache"]:
        return {"q": dr.tokens((sum(q), H, d)).to(dt), "k": dr.tokens((rows, Hk, d)).to(dt), "v": dr.tokens((rows, Hk, d)).to(dt)}
    x = dr.tokens((rows, H + 2 * Hk, d)).to(dt)
    return {"q": x[:, :H], "k": x[:, H:H + Hk], "v": x[:, H + Hk:]}


def prepare(case, seed):
    s, op = _inputs(case, seed), case["op"]
    s["case"] = case
    if op in ("quantize", "linear"):
        rows, K = s["x"].shape
        s["xq"] = torch.empty(rows * _up(K, 256) * 128, dtype=torch.uint8, device="cuda")
        s["xs"] = torch.empty(rows * _up(K, 512) * 16, dtype=torch.uint8, device="cuda")
        s["y"] = torch.empty((rows, K if op == "quantize" else case["N"]), dtype=_dtype(case.get("out", "bf16")), device="cuda")
    elif op == "rope":
        s["w"] = _frequencies(case)
        s["y"] = torch.empty_like(s["x"])
    else:
        s["o"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    if own and op == "rope":
        from paper_2510_01565_amd import dit
        s["w"] = dit.rope_frequencies(case["rot"], THETA, case["factor"], ORIGINAL, LOW, HIGH)
    if own and op == "attention":
        from paper_2510_01565_amd import dit
        s["seqs"] = dit.Sequences(*_lengths(case), _slots(case)[0])
        s["wsb"] = dit.attention_grouped_workspace_size(s["seqs"], case["heads"], case["kv_heads"], case["d"],
                                                        dit.DIT_BF16 if case["dtype"] == "bf16" else dit.DIT_F32)
        s["scratch"] = torch.empty(s["wsb"], dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------- plain forms
def _bits(byte):
    """2^(byte - 127) in 32 bits, exactly."""
    return (byte.int() << 23).view(torch.float32)


def _quantize(x):
    """Values on the e2m1 grid [rows, blocks, 32] and scale bytes [rows, blocks] (exponent + 127)."""
    rows, K = x.shape
    t = torch.nn.functional.pad(x.float(), (0, _up(K, BLOCK) * BLOCK - K)).view(rows, -1, BLOCK)
    a = t.abs().amax(dim=2)
    m, e = torch.frexp(a)                              # a = m 2^e, m in [0.5, 1); 6 = 0.75 * 2^3
    byte = (e - 3 + (m > 0.75).int() + 127).clamp(0, 254)
    byte = torch.where(a == 0, 127, byte).int()
    v = t * _bits(254 - byte)[:, :, None]
    _, e = torch.frexp(v)
    step = _bits((e - 1).clamp(min=0) + 126)           # of the grid at v: 0.5 up to 2, then 1, then 2
    return torch.round(v / step) * step, byte


def _values(v, byte, K):
    return (v * _bits(byte)[:, :, None]).view(v.shape[0], -1)[:, :K]


def _pack(v, byte):
    """Codes, two to a byte, the lower nibble first, rows of ceil(K / 256) * 128 bytes; scale bytes in rows of ceil(K / 512) * 16,
    the sixteen of 512 elements as four times four: block 4 s + g at 4 g + s."""
    rows, nb = byte.shape
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=v.device)
    code = torch.bucketize(v.abs(), grid) + 8 * torch.signbit(v)
    code = torch.nn.functional.pad(code.view(rows, -1), (0, (_up(nb, 8) * 8 - nb) * BLOCK)).to(torch.uint8)
    s = torch.nn.functional.pad(byte, (0, _up(nb, 16) * 16 - nb), value=127).to(torch.uint8)
    return code[:, 0::2] | code[:, 1::2] << 4, s.view(rows, -1, 4, 4).transpose(2, 3).reshape(rows, -1).contiguous()


def _unpack(q, s, K):
    """What packed codes and scales stand for, [rows, K]."""
    rows = q.shape[0]
    code = torch.stack([q & 15, q >> 4], dim=2).view(rows, -1, BLOCK).int()
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=q.device)[code & 7]
    byte = s.view(rows, -1, 4, 4).transpose(2, 3).reshape(rows, -1)[:, : v.shape[1]]
    return _values(torch.where(code >= 8, -v, v), byte, K)


def _rope(case, x, pos, w):
    """The rotation in 32 bits, with angles in 64."""
    rot = case["rot"]
    angle = pos.double()[:, None] * torch.tensor(w, dtype=torch.float64, device=x.device)
    c, s = ((_magnitude(case) * f(angle)).float()[:, None, :] for f in (torch.cos, torch.sin))
    t = x[:, :, :rot].float()
    a, b = (t[:, :, : rot // 2], t[:, :, rot // 2:]) if case["layout"] == "half" else (t[:, :, 0::2], t[:, :, 1::2])
    y = torch.cat([a * c - b * s, a * s + b * c], 2) if case["layout"] == "half" else \
        torch.stack([a * c - b * s, a * s + b * c], 3).view(t.shape)
    return torch.cat([y.to(x.dtype), x[:, :, rot:]], 2)


def _attention(case, q, k, v):
    """Sequence by sequence and key head by key head, all scores at once, softmax in 32 bits."""
    ql, kl = _lengths(case)
    first, _ = _slots(case)
    H, Hk, d = case["heads"], case["kv_heads"], case["d"]
    G = H // Hk
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    at = 0
    for n, m, f in zip(ql, kl, first):
        seen = torch.arange(m, device=q.device)[None, :] <= torch.arange(m - n, m, device=q.device)[:, None]
        for h in range(Hk):
            qs = q[at:at + n, h * G:(h + 1) * G].float().transpose(0, 1).reshape(G * n, d)
            s = torch.matmul(qs, k[f:f + m, h].float().t().contiguous()) / math.sqrt(d)
            s = s.view(G, n, m)
            if case["causal"]:
                s = s.masked_fill_(~seen, float("-inf"))
            top = s.amax(2, keepdim=True)
            p = torch.exp(s.sub_(torch.where(torch.isinf(top), 0.0, top)))
            total = p.sum(2, keepdim=True)
            r = torch.matmul(p.view(G * n, m), v[f:f + m, h].float()).view(G, n, d) / torch.where(total == 0, 1.0, total)
            o[at:at + n, h * G:(h + 1) * G] = r.transpose(0, 1).to(o.dtype)
        at += n
    return o


# ---------------------------------------------------------------------------- one pass
def run(s):
    case, op = s["case"], s["case"]["op"]
    if not own:
        if op == "quantize":
            return _values(*_quantize(s["x"]), case["K"]).to(torch.bfloat16)
        if op == "linear":
            y = torch.matmul(_values(*_quantize(s["x"]), case["K"]), _unpack(s["wq"], s["ws"], case["K"]).t())
            if s["b"] is not None:
                y += s["b"].float()
            return y.to(_dtype(case["out"]))
        if op == "rope":
            return _rope(case, s["x"], s["pos"], s["w"])
        return _attention(case, s["q"], s["k"], s["v"])
    from paper_2510_01565_amd import dit
    dt = dit.DIT_BF16 if case.get("dtype", "bf16") == "bf16" else dit.DIT_F32
    if op == "quantize":
        dit.dit_quantize_fp4(case["rows"], case["K"], dt, s["x"], s["xq"], s["xs"])
        dit.dit_dequantize_fp4(case["rows"], case["K"], s["xq"], s["xs"], dit.DIT_BF16, s["y"])
        return s["y"]
    if op == "linear":
        dit.dit_quantize_fp4(case["M"], case["K"], dit.DIT_BF16, s["x"], s["xq"], s["xs"])
        dit.dit_linear_fp4(case["M"], case["N"], case["K"], s["xq"], s["xs"], s["wq"], s["ws"], s["b"], dit.DIT_BF16, s["y"],
                           dit.DIT_BF16 if case["out"] == "bf16" else dit.DIT_F32)
        return s["y"]
    if op == "rope":
        dit.dit_rope(case["rows"], case["heads"], case["d"], case["rot"], dit.DIT_ROPE_HALF if case["layout"] == "half" else
                     dit.DIT_ROPE_PAIRS, dt, s["pos"], s["w"], _magnitude(case), s["x"], case["heads"] * case["d"], s["y"],
                     case["heads"] * case["d"])
        return s["y"]
    H, Hk, d = case["heads"], case["kv_heads"], case["d"]
    dit.dit_attention_grouped(s["seqs"], H, Hk, d, dt, dit.DIT_CAUSAL if case["causal"] else 0, 1.0 / math.sqrt(d), s["q"],
                              s["q"].stride(0), s["k"], s["v"], s["k"].stride(0), s["o"], H * d, s["scratch"], s["wsb"])
    return s["o"]


# ---------------------------------------------------------------------------- 64 bits
def _pow2(e):
    """2^e in 64 bits from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(x):
    """x in blocks of 32 on the nearest value of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale, ties to the even code."""
    rows, K = x.shape
    t = torch.nn.functional.pad(x.double(), (0, _up(K, BLOCK) * BLOCK - K)).view(rows, -1, BLOCK)
    a = t.abs().amax(dim=2, keepdim=True)
    e = torch.floor(torch.log2(torch.where(a > 0, a / 6.0, 1.0)))  # the smallest with 6 2^e >= a, but for log2's last place
    e = torch.where(_pow2(e) * 6.0 < a, e + 1, e)
    e = torch.where(_pow2(e - 1) * 6.0 >= a, e - 1, e).clamp(min=-127.0)
    scale = _pow2(torch.where(a > 0, e, 0.0))
    v = t.abs() / scale
    grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    out = torch.zeros_like(v)
    for i in range(1, 8):
        mid = (grid[i - 1] + grid[i]) / 2
        out = torch.where((v > mid) | ((v == mid) & (i % 2 == 0)), grid[i], out)
    return (torch.copysign(out, t) * scale).view(rows, -1)[:, :K]


def _exact_weights(q, s, K):
    """Element by element: (-1)^sign m 2^e of its nibble's bits, times the scale of its block."""
    at = torch.arange(K, device=q.device)
    n = (q[:, at // 2].long() >> (at % 2 * 4)) & 15
    e, m = n >> 1 & 3, n & 1
    v = torch.where(e == 0, 0.5 * m.double(), (1 + 0.5 * m.double()) * _pow2((e - 1).clamp(min=0)))
    b = at // BLOCK
    scale = _pow2(s[:, b // 16 * 16 + b % 4 * 4 + b // 4 % 4].long() - 127)
    return torch.where(n >= 8, -v, v) * scale


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "quantize":
        return _exact_values(s["x"])
    if op == "linear":
        w = _exact_weights(s["wq"], s["ws"], case["K"])
        y = torch.matmul(_exact_values(s["x"]), w.t().contiguous())
        return y if s["b"] is None else y + s["b"].double()
    if op == "rope":
        # as complex numbers
        rot, x = case["rot"], s["x"].double()
        turn = torch.polar(torch.full((1, 1), _magnitude(case), dtype=torch.float64, device="cuda"),
                           s["pos"].double()[:, None] * torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda"))
        at = torch.arange(rot, device="cuda").view(2, -1) if case["layout"] == "half" else torch.arange(rot, device="cuda").view(-1, 2).t()
        z = torch.complex(x[:, :, at[0]], x[:, :, at[1]]) * turn[:, None, :]
        x[:, :, at[0]], x[:, :, at[1]] = z.real, z.imag
        return x
    ql, kl = _lengths(case)
    first, _ = _slots(case)
    H, G, d = case["heads"], case["heads"] // case["kv_heads"], case["d"]
    o, at = torch.zeros((sum(ql), H, d), dtype=torch.float64, device="cuda"), 0
    for n, m, f in zip(ql, kl, first):
        for h in range(H):
            k, v = s["k"][f:f + m, h // G].double(), s["v"][f:f + m, h // G].double()
            for i in range(0, n, 4096):
                r = min(n, i + 4096)
                most = m - n + r if case["causal"] else m
                c = torch.matmul(s["q"][at + i:at + r, h].double(), k[:most].t().contiguous()) / math.sqrt(d)
                if case["causal"]:
                    c += torch.triu(torch.full_like(c, float("-inf")), diagonal=m - n + i + 1)
                o[at + i:at + r, h] = torch.matmul(torch.softmax(c, dim=1), v[:most])
        at += n
    return o


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    op, es = case["op"], 2 if case.get("dtype", "bf16") == "bf16" else 4
    if op == "quantize":
        rows, K = case["rows"], case["K"]
        return {"bytes": rows * K * es + rows * _up(K, BLOCK) * 17 + rows * K * 2, "flops": 2 * rows * K}
    if op == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        b = M * K * 2 + N * _up(K, BLOCK) * 17 + M * N * (2 if case["out"] == "bf16" else 4) + (2 * N if case["bias"] else 0)
        return {"bytes": b, "flops": 2 * M * N * K}
    if op == "rope":
        n = case["rows"] * case["heads"] * case["d"]
        return {"bytes": 2 * n * es + 4 * case["rows"], "flops": 3 * case["rows"] * case["heads"] * case["rot"]}
    q, kv = _lengths(case)
    pairs = sum(n * m - (n * (n - 1) // 2 if case["causal"] else 0) for n, m in zip(q, kv))
    return {"bytes": (2 * sum(q) * case["heads"] + 2 * sum(kv) * case["kv_heads"]) * case["d"] * es,
            "flops": 4 * pairs * case["heads"] * case["d"]}
