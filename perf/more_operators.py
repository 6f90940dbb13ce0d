"""Operators around a cache in 4 bits: the calls, their plain forms and their definitions.

Kinds:

  turn      norms of the queries' and keys' heads with the position rotation in the same pass
  turn_grad its backward pass: gradients of queries, keys and of the norms' weights and biases
  append4   new tokens of a batch of requests into the pages of a 4-bit cache, normalised and
            rotated on the way, and what the cache then holds for them
  attn4     attention of a batch of requests over the pages of a 4-bit cache, with its
            log-sum-exp

The cache holds 32 values of a head of a token as one power of two and 32 four-bit numbers:
sign and 0, 0.5, 1, 1.5, 2, 3, 4, 6. The power is the smallest with no value above 7 times
it, and values are rounded to nearest, ties to the even code. A page has for every key head
[page rows, head_dim / 2] bytes of keys (the even value in the low half of a byte), as many of
values, and [page rows, 2, head_dim / 32] exponents (plus 127) of the keys' and the values'
powers.

``own`` selects this package's kernels; otherwise elementary torch operations in fp32
(angles and whatever is rounded to 4 bits in fp64), rounded once at the end.
"""

import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DTYPES = {"bf16": BF16, "f32": F32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-6
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one token each of 64 requests, weights on the norms, far into a scaled context: all latency
        {"name": "turn_tokens", "kind": "turn", "rows": 64, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "rotary_dim": 128, "axes": 1, "interleaved": False, "scaling": "parts", "norm": "rms", "weight": True,
         "bias": False, "x": "bf16", "packed": True},
        # a chunk of three latent frames at the 14B shape, q and k columns of one wider product
        {"name": "turn_chunk_14b", "kind": "turn", "rows": 4680, "heads": 40, "kv_heads": 40, "head_dim": 128,
         "rotary_dim": 128, "axes": 3, "interleaved": True, "scaling": "none", "norm": "rms", "weight": True,
         "bias": False, "x": "bf16", "packed": True},
        # the backward pass of the 1.3B chunk
        {"name": "turn_grad_1p3b", "kind": "turn_grad", "rows": 4680, "heads": 12, "kv_heads": 12, "head_dim": 128,
         "rotary_dim": 128, "axes": 3, "interleaved": True, "scaling": "none", "norm": "rms", "weight": True,
         "bias": False, "x": "bf16", "packed": False},
        # an odd count of rows of few narrow heads in fp32, centred norms with biases, part of each head turned
        {"name": "turn_grad_odd", "kind": "turn_grad", "rows": 1001, "heads": 9, "kv_heads": 3, "head_dim": 96,
         "rotary_dim": 48, "axes": 1, "interleaved": False, "scaling": "none", "norm": "layer", "weight": True,
         "bias": True, "x": "f32", "packed": False},
        # one token each of 64 requests into their pages: all latency
        {"name": "append4_tokens", "kind": "append4", "requests": 64, "most": 1, "pad": 3, "page": 64, "pages": 16,
         "sink": 0, "window": 0, "first": 1000003, "heads": 32, "kv_heads": 8, "head_dim": 128, "rotary_dim": 128,
         "axes": 1, "interleaved": False, "scaling": "parts", "norm": "rms"},
        # a latent frame of four forked rollouts into rings of sink and recent keys, no norm
        {"name": "append4_frames", "kind": "append4", "requests": 4, "most": 1560, "pad": 0, "page": 256, "pages": 19,
         "sink": 1560, "window": 3304, "first": 0, "heads": 12, "kv_heads": 12, "head_dim": 128, "rotary_dim": 128,
         "axes": 3, "interleaved": True, "scaling": "none", "norm": "none"},
        # the smallest batch of the parity tests' head shape: all latency
        {"name": "attn4_tiny", "kind": "attn4", "requests": 2, "most": 1, "pad": 0, "page": 32, "pages": 8,
         "heads": 2, "kv_heads": 2, "head_dim": 64, "out": "bf16"},
        # one stream's single token against the whole history of seven chunks
        {"name": "attn4_alone", "kind": "attn4", "requests": 1, "most": 1, "pad": 0, "page": 4096, "pages": 8,
         "heads": 12, "kv_heads": 12, "head_dim": 128, "out": "f32"},
        # single tokens of 64 requests of very different lengths, four query heads to a key head
        {"name": "attn4_tokens", "kind": "attn4", "requests": 64, "most": 1, "pad": 3, "page": 64, "pages": 256,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "out": "bf16"},
        # a few tokens each of three requests behind very long contexts
        {"name": "attn4_long", "kind": "attn4", "requests": 3, "most": 5, "pad": 0, "page": 128, "pages": 1024,
         "heads": 32, "kv_heads": 8, "head_dim": 128, "out": "bf16"},
        # middling runs of rows of many requests, narrow heads
        {"name": "attn4_runs", "kind": "attn4", "requests": 24, "most": 77, "pad": 5, "page": 32, "pages": 129,
         "heads": 16, "kv_heads": 8, "head_dim": 64, "out": "bf16"},
        # a chunk of three latent frames at the 1.3B shape against the whole history of seven chunks
        {"name": "attn4_chunk", "kind": "attn4", "requests": 1, "most": 4680, "pad": 0, "page": 4096, "pages": 8,
         "heads": 12, "kv_heads": 12, "head_dim": 128, "out": "bf16"},
    ]


# a drawn case costs no more than the largest listed one of its kind, in operations, in
# weights of the plain form and in keys
MOST_ATTN = 4 * 4680 * 32768 * 1536
MOST_WEIGHTS = 4680 * 12 * 32768
MOST_VALUES = 2 * 4680 * 5120
MOST_CACHE = 3 * 1024 * 128 * 8 * 128


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / step)) * step))


def _heads(rng):
    kv = rng.choice((1, 2, 3, 4, 8, 12, 16))
    return kv * rng.choice((1, 1, 2, 3, 4, 8) if kv < 8 else (1, 1, 2, 4)), kv


def _turned(rng, head_dim):
    axes = rng.choice((1, 1, 3))
    part = head_dim if axes == 3 or head_dim % 32 else rng.choice((head_dim, head_dim, head_dim // 2))
    return {"head_dim": head_dim, "rotary_dim": part, "axes": axes, "interleaved": rng.random() < 0.5,
            "scaling": "none" if axes == 3 else rng.choice(("none", "linear", "base", "parts"))}


def draw(rng):
    kind = rng.choice(("turn", "turn_grad", "append4", "attn4", "attn4", "attn4"))
    if kind in ("turn", "turn_grad"):
        heads, kv = _heads(rng)
        head_dim = rng.choice((32, 64, 80, 96, 128, 128, 128, 256))
        rows = _log(rng, 1, min(16384, MOST_VALUES // ((heads + kv) * head_dim)))
        return {"kind": kind, "rows": rows, "heads": heads, "kv_heads": kv, **_turned(rng, head_dim),
                "norm": rng.choice(("rms", "rms", "layer")), "weight": rng.random() < 0.8, "bias": rng.random() < 0.3,
                "x": rng.choice(("bf16", "bf16", "f32")), "packed": rng.random() < 0.5}
    while True:
        heads, kv = _heads(rng)
        head_dim = rng.choice((64, 128, 128))
        requests = _log(rng, 1, 128)
        most = rng.choice((1, rng.randint(1, 8), _log(rng, 1, 4680)))
        page = 1 << rng.randint(5, 12)
        c = {"kind": kind, "requests": requests, "most": most, "pad": rng.choice((0, 0, rng.randint(1, 9))),
             "page": page, "pages": max(1, _log(rng, 32, 131072) // page), "heads": heads, "kv_heads": kv}
        capacity = c["page"] * c["pages"]
        if kind == "append4":
            ring = rng.random() < 0.4
            if (most <= capacity <= 16384 and requests * capacity * kv * head_dim <= MOST_CACHE
                    and requests * most * (heads + 2 * kv) * head_dim <= MOST_VALUES):
                sink = rng.randint(0, capacity // 4) if ring else 0
                turned = _turned(rng, head_dim)
                return {**c, "sink": sink, "window": capacity - sink if ring else 0,
                        "first": 0 if turned["axes"] == 3 else rng.choice((0, _log(rng, 1, 2000000))), **turned,
                        "norm": rng.choice(("none", "rms", "rms", "layer"))}
            continue
        rows = requests * most
        if (rows * heads * capacity <= MOST_WEIGHTS and 4 * rows * heads * head_dim * capacity <= MOST_ATTN
                and requests * capacity * kv * head_dim <= MOST_CACHE):
            return {**c, "head_dim": head_dim, "out": rng.choice(("bf16", "bf16", "f32"))}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + 31)
    return g


def _randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=F32).to(dtype)


def _randint(g, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)


def _lengths(c, g):
    """Rows of each request (the first one `most`, now and then none) and their running sum."""
    n = _randint(g, 1 if c["most"] == 1 else 0, c["most"] + 1, c["requests"])
    n[0] = c["most"]
    start = torch.zeros(c["requests"] + 1, dtype=torch.int32, device="cuda")
    start[1:] = torch.cumsum(n, 0)
    return n, start


def _rows(c):
    """Rows of the batch's tensors: room for every request's most, and padding."""
    return c["requests"] * c["most"] + c["pad"]


def _frequencies(c):
    """Each pair's radians per position (fp64), the pairs of each axis, the axis of each pair, the factor of cos and sin."""
    half = c["rotary_dim"] // 2
    side = half // 3
    axes = (half - 2 * side, side, side) if c["axes"] == 3 else (half,)
    base, f = 10000.0, []
    for n in axes:
        j = torch.arange(n, dtype=F64)
        b = base * 8.0 ** (n / (n - 1.0)) if c["scaling"] == "base" else base
        f.append(b ** (-j / n))
    f = torch.cat(f)
    amplitude = 1.0
    if c["scaling"] == "linear":
        f = f / 4.0
    if c["scaling"] == "parts":  # fast pairs as they are, slow ones slowed down, a ramp between
        lo, hi = (half * math.log(4096 / (b * 2 * math.pi)) / math.log(base) for b in (32.0, 1.0))
        lo, hi = max(0.0, math.floor(lo)), math.ceil(hi)
        ramp = ((torch.arange(half, dtype=F64) - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        f = f * (1 - ramp) + f / 16.0 * ramp
        amplitude = 1.25
    axis = torch.tensor([k for k, n in enumerate(axes) for _ in range(n)])
    return {"f": f.cuda(), "axes": axes, "axis": axis.cuda(), "amplitude": amplitude}


def _positions(c, g, rows):
    if c["axes"] == 3:  # frames of 30 x 52 places from some frame of a long video on
        r = torch.arange(rows, device="cuda", dtype=torch.int32)
        t0 = _randint(g, 0, 400, 1)
        return torch.stack((t0 + r // 1560, r % 1560 // 52, r % 52), dim=1).contiguous()
    return _randint(g, 0, 200000, rows, 1)


def _weights(c, g):
    s = {"q_weight": None, "k_weight": None, "q_bias": None, "k_bias": None}
    for name in ("q", "k"):
        if c.get("weight", c["norm"] != "none"):
            s[name + "_weight"] = 1 + 0.2 * _randn(g, c["head_dim"])
        if c.get("bias"):
            s[name + "_bias"] = 0.1 * _randn(g, c["head_dim"])
    return s


def _projected(c, g, rows, dtype, packed=True):
    """q, k and v: columns of one product with the rows of all three, or tensors of their own."""
    d = c["head_dim"]
    hidden, kv = c["heads"] * d, c["kv_heads"] * d
    wide = _randn(g, rows, hidden + 2 * kv, dtype=dtype)
    q, k, v = wide[:, :hidden], wide[:, hidden:hidden + kv], wide[:, hidden + kv:]
    return (q, k, v) if packed else (q.contiguous(), k.contiguous(), v.contiguous())


def _table(c, g):
    """The pages of each request, in no order, out of a pool with some more."""
    n = c["requests"] * c["pages"]
    pages = torch.randperm(n + 3, generator=g, device="cuda")[:n].to(torch.int32)
    return pages.view(c["requests"], c["pages"]).contiguous(), n + 3


def _page_bytes(c):
    return c["page"] * (c["head_dim"] + c["head_dim"] // 16)


def _filled(c, g, n_pages):
    """Pages that hold normally distributed keys and values."""
    kv, p, d = c["kv_heads"], c["page"], c["head_dim"]
    cache = torch.empty(n_pages, kv, _page_bytes(c), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (kv * p * d))
    for at in range(0, n_pages, step):  # some at a time, for the room that it takes
        n = min(step, n_pages - at)
        scales = []
        for i in range(2):
            # heads of different spread, and keys with a few large channels
            x = _randn(g, n, kv, p, d) * (0.6 + 0.8 * torch.rand(1, kv, 1, 1, generator=g, device="cuda"))
            if i == 0:
                x = x * torch.where(torch.rand(d, generator=g, device="cuda") < 0.05, 3.0, 1.0)
            codes, power = _to_codes(x)
            codes = codes.to(torch.uint8)
            cache[at:at + n, :, i * p * d // 2:(i + 1) * p * d // 2] = (codes[..., 0::2] | codes[..., 1::2] << 4).flatten(2)
            scales.append((power + 127).to(torch.uint8))
        cache[at:at + n, :, p * d:] = torch.stack(scales, dim=3).flatten(2)
    return cache


def prepare(case, seed):
    c, g = case, _gen(seed)
    if c["kind"] in ("turn", "turn_grad"):
        q, k, _ = _projected(c, g, c["rows"], DTYPES[c["x"]], c["packed"])
        s = {"c": c, **_frequencies(c), "positions": _positions(c, g, c["rows"]), "q": q, "k": k, **_weights(c, g)}
        if c["kind"] == "turn_grad":
            s["d_q"], s["d_k"], _ = _projected(c, g, c["rows"], DTYPES[c["x"]], False)
        return s
    rows = _rows(c)
    n, start = _lengths(c, g)
    table, n_pages = _table(c, g)
    capacity = c["page"] * c["pages"]
    if c["kind"] == "append4":
        before = _randint(g, 0, 3 * capacity, c["requests"]) if c["window"] else (
            _randint(g, 0, 1 << 30, c["requests"]) % (capacity - n + 1).to(torch.int32))
        q, k, v = _projected(c, g, rows, BF16)
        return {"c": c, **_frequencies(c), **_weights(c, g), "start": start, "before": before, "q": q, "k": k, "v": v,
                "positions": _positions(c, g, rows) if c["axes"] == 3 else None, "table": table,
                "cache": torch.zeros(n_pages, c["kv_heads"], _page_bytes(c), dtype=torch.uint8, device="cuda"),
                "q_out": torch.zeros(rows, c["heads"] * c["head_dim"], dtype=BF16, device="cuda")}
    lens = _randint(g, 0, capacity + 1, c["requests"])  # keys, none among them now and then
    lens[0] = capacity - capacity // 4096  # (32760 of 32768)
    hidden = c["heads"] * c["head_dim"]
    return {"c": c, "start": start, "lens": lens, "q": _randn(g, rows, hidden, dtype=BF16), "table": table,
            "cache": _filled(c, g, n_pages),
            "out": torch.zeros(rows, hidden, dtype=DTYPES[c["out"]], device="cuda"),
            "lse": torch.zeros(c["heads"], rows, dtype=F32, device="cuda")}


# ------------------------------------------------------------------ plain forms
def _normed(x, norm):
    """The normalised last dimension and the reciprocal deviations."""
    if norm == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    return x * r, r


def _turn(x, positions, s, inverse=False):
    """x [rows, heads, head_dim] with each head's first rotary_dim values turned, in x's type."""
    c = s["c"]
    angle = positions.double()[:, s["axis"]] * s["f"]
    cos = (angle.cos() * s["amplitude"]).to(x.dtype)[:, None, :]
    sin = (angle.sin() * (-s["amplitude"] if inverse else s["amplitude"])).to(x.dtype)[:, None, :]
    t, rest = x[..., :c["rotary_dim"]], x[..., c["rotary_dim"]:]
    half = c["rotary_dim"] // 2
    if c["interleaved"]:
        a, b = t[..., 0::2], t[..., 1::2]
        t = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = t[..., :half], t[..., half:]
        t = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((t, rest), dim=-1)


def _plain_heads(x, weight, bias, positions, s, dtype):
    """x [rows, heads * head_dim], every head normalised and turned, as [rows, heads, head_dim] of `dtype`."""
    c = s["c"]
    x = x.to(dtype).view(x.shape[0], -1, c["head_dim"])
    if c["norm"] != "none":
        x = _normed(x, c["norm"])[0]
    if weight is not None:
        x = x * weight.to(dtype)
    if bias is not None:
        x = x + bias.to(dtype)
    return _turn(x, positions, s)


def _plain_turn(s):
    q = _plain_heads(s["q"], s["q_weight"], s["q_bias"], s["positions"], s, F32)
    k = _plain_heads(s["k"], s["k_weight"], s["k_bias"], s["positions"], s, F32)
    return q.flatten(1).to(s["q"].dtype), k.flatten(1).to(s["k"].dtype)


def _plain_back(name, s):
    c, out = s["c"], {}
    x = s[name].float().view(c["rows"], -1, c["head_dim"])
    d = _turn(s["d_" + name].float().view(x.shape), s["positions"], s, inverse=True)
    xhat, r = _normed(x, c["norm"])
    if s[name + "_bias"] is not None:
        out[name + "_bias"] = d.sum(dim=(0, 1))
    if s[name + "_weight"] is not None:
        out[name + "_weight"] = (d * xhat).sum(dim=(0, 1))
        d = d * s[name + "_weight"]
    back = d - xhat * (d * xhat).mean(dim=-1, keepdim=True)
    if c["norm"] == "layer":
        back = back - d.mean(dim=-1, keepdim=True)
    out[name] = (back * r).flatten(1).to(s[name].dtype)
    return out


def _to_codes(x):
    """Codes of x's values (last dimension, in blocks of 32) and the blocks' powers of two."""
    blocks = x.unflatten(-1, (-1, 32))
    top, power = torch.frexp(blocks.abs().amax(dim=-1))  # the largest value is top 2^power, top in [0.5, 1)
    power = (power - 3 + (top > 0.875).to(power.dtype)).clamp(-120, 125)
    y = torch.ldexp(blocks, -power[..., None])
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return (code + 8 * (y < 0)).flatten(-2), power


def _from_codes(codes, power):
    """Codes [..., n, d] and powers [..., n, d / 32] as fp32 values."""
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    return (grid[codes.int()].unflatten(-1, (-1, 32)) * torch.exp2(power.float())[..., None]).flatten(-2)


def _requests_of(start, rows):
    """The request of each row (the count of requests for rows behind the last) and its place in it."""
    r = torch.arange(rows, device="cuda", dtype=torch.int32)
    b = (r[:, None] >= start[None, 1:]).sum(dim=1)
    return b, r - start[b]


def _plain_append4(s):
    c, rows, capacity = s["c"], _rows(s["c"]), s["c"]["page"] * s["c"]["pages"]
    b, i = _requests_of(s["start"], rows)
    new = s["start"][1:] - s["start"][:-1]
    real = b < c["requests"]
    bb = b.clamp(max=c["requests"] - 1)
    at = s["before"][bb] + i
    place = at.long()
    kept = real
    if c["window"]:
        place = torch.where(place < c["sink"], place, c["sink"] + (place - c["sink"]) % c["window"])
        kept = kept & ((at < c["sink"]) | (new[bb] - i <= c["window"]))
    positions = torch.where(real, c["first"] + at, torch.zeros_like(at)).to(torch.int32)[:, None]
    if s["positions"] is not None:
        positions = s["positions"]
    q = _plain_heads(s["q"], s["q_weight"], s["q_bias"], positions, s, F32).flatten(1).to(BF16)
    s["q_out"][:] = torch.where(real[:, None], q, s["q_out"])
    # what is rounded to 4 bits, in fp64: a value next to a border keeps its side
    k = _plain_heads(s["k"], s["k_weight"], s["k_bias"], positions, s, F64)
    v = s["v"].double().view(rows, -1, c["head_dim"])
    place = torch.where(kept, place, torch.zeros_like(place))
    page, row = s["table"][bb, place // c["page"]].long(), place % c["page"]
    kv, p, d = c["kv_heads"], c["page"], c["head_dim"]
    back = []
    scales = s["cache"][:, :, p * d:].unflatten(2, (p, 2, d // 32))
    for n, x in enumerate((k, v)):
        codes, power = _to_codes(x)
        codes, power = codes[kept].to(torch.uint8), (power[kept] + 127).to(torch.uint8)
        held = s["cache"][:, :, n * p * d // 2:(n + 1) * p * d // 2].unflatten(2, (p, d // 2))
        at = (page[kept][:, None], torch.arange(kv, device="cuda")[None, :], row[kept][:, None])
        held[at] = codes[..., 0::2] | codes[..., 1::2] << 4
        scales[at + (torch.full_like(at[0], n),)] = power
        # and read back for every row that has a place
        h = held[page[:, None], at[1], row[:, None]]
        e = scales[page[:, None], at[1], row[:, None], n].float() - 127
        x = _from_codes(torch.stack((h & 15, h >> 4), dim=-1).flatten(-2), e)
        back.append(torch.where(kept[:, None, None], x, torch.zeros_like(x)).flatten(1).to(BF16))
    return back[0], back[1]


def _plain_attn4(s):
    c, rows = s["c"], _rows(s["c"])
    n, m, d, kv, p = c["requests"], c["most"], c["head_dim"], c["kv_heads"], c["page"]
    g, capacity = c["heads"] // kv, c["page"] * c["pages"]
    b, i = _requests_of(s["start"], rows)
    at = torch.where(b < n, b * m + i, torch.full_like(b, n * m))
    q = torch.zeros(n * m + 1, c["heads"] * d, device="cuda")
    q[at] = s["q"].float()  # rows behind the last request meet in one more row
    q = q[:-1].view(n, m, kv, g, d).permute(0, 2, 1, 3, 4).reshape(n, kv, m * g, d) * (1.0 / math.sqrt(d))
    held = s["cache"][s["table"].long()].transpose(1, 2)  # [n, kv, pages, bytes]
    scales = held[..., p * d:].unflatten(3, (p, 2, d // 32)).flatten(2, 3).float() - 127
    codes = held[..., :p * d // 2].unflatten(3, (p, d // 2)).flatten(2, 3)
    k = _from_codes(torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2), scales[:, :, :, 0])
    codes = held[..., p * d // 2:p * d].unflatten(3, (p, d // 2)).flatten(2, 3)
    v = _from_codes(torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2), scales[:, :, :, 1])
    w = torch.matmul(q, k.transpose(2, 3).contiguous())
    seen = torch.arange(capacity, device="cuda")[None, :] < s["lens"][:, None]
    w.masked_fill_(~seen[:, None, None, :], -math.inf)
    top = w.amax(dim=3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    w = w.sub_(top).exp_()
    total = w.sum(dim=3, keepdim=True)
    o = torch.matmul(w, v)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (top + total.log())[..., 0]
    o = o.view(n, kv, m, g, d).permute(0, 2, 1, 3, 4).reshape(n * m, -1)
    lse = lse.view(n, kv, m, g).permute(1, 3, 0, 2).reshape(c["heads"], n * m)
    real, at = b < n, at.clamp(max=n * m - 1)
    s["out"][:] = torch.where(real[:, None], o[at].to(s["out"].dtype), s["out"])
    s["lse"][:] = torch.where(real[None, :], lse[:, at], s["lse"])
    return s["out"], s["lse"]


# ------------------------------------------------------------------ the calls
def _own_turn(s):
    import paper_2607_00712_amd as ispa
    c = s["c"]
    return ispa.norm_rotary(s["q"], s["k"], s["positions"], s["f"], c["heads"], n_kv_heads=c["kv_heads"],
                            norm=c["norm"], q_weight=s["q_weight"], k_weight=s["k_weight"], q_bias=s["q_bias"],
                            k_bias=s["k_bias"], eps=EPS, axes=s["axes"], interleaved=c["interleaved"],
                            amplitude=s["amplitude"])


def _own_turn_grad(s):
    import paper_2607_00712_amd as ispa
    c = s["c"]
    return ispa.norm_rotary_backward(s["d_q"], s["d_k"], s["q"], s["k"], s["positions"], s["f"], c["heads"],
                                     n_kv_heads=c["kv_heads"], norm=c["norm"], q_weight=s["q_weight"],
                                     k_weight=s["k_weight"], q_bias=s["q_bias"], k_bias=s["k_bias"], eps=EPS,
                                     axes=s["axes"], interleaved=c["interleaved"], amplitude=s["amplitude"])


def _own_append4(s):
    import paper_2607_00712_amd as ispa
    c = s["c"]
    slots, positions, _ = ispa.slot_map(s["start"], s["before"], c["page"] * c["pages"], _rows(c), sink=c["sink"],
                                        window=c["window"], first_position=c["first"])
    at = positions if s["positions"] is None else s["positions"]
    ispa.kv4_append(s["q"], s["k"], s["v"], at, slots, s["f"], c["heads"], s["cache"], s["table"],
                    n_kv_heads=c["kv_heads"], norm=c["norm"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                    axes=s["axes"], interleaved=c["interleaved"], amplitude=s["amplitude"], q_out=s["q_out"],
                    q_start=s["start"])
    return ispa.kv4_read(s["cache"], s["table"], slots, c["head_dim"])


def _own_attn4(s):
    import paper_2607_00712_amd as ispa
    c = s["c"]
    return ispa.attn_kv4(s["q"], s["cache"], s["table"], s["start"], s["lens"], c["heads"], max_q=c["most"],
                         out=s["out"], lse=s["lse"])


def run(state):
    s, kind = state, state["c"]["kind"]
    if kind == "turn":
        q, k = _own_turn(s) if own else _plain_turn(s)
        return {"q": q, "k": k}
    if kind == "turn_grad":
        return _own_turn_grad(s) if own else {**_plain_back("q", s), **_plain_back("k", s)}
    if kind == "append4":
        k, v = _own_append4(s) if own else _plain_append4(s)
        return {"q": s["q_out"], "k": k, "v": v}
    out, lse = _own_attn4(s) if own else _plain_attn4(s)
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------ definitions, in 64 bits
def _exact_heads(x, weight, bias, positions, s):
    """[rows, heads, head_dim]: normalised heads, their pairs as complex numbers times a unit number."""
    c, half, f = s["c"], s["c"]["rotary_dim"] // 2, s["f"].cpu().tolist()
    x = x.reshape(len(x), -1, c["head_dim"])
    if c["norm"] == "layer":
        x = (x - x.mean(2, keepdim=True)) / (x.var(2, unbiased=False, keepdim=True) + EPS).sqrt()
    elif c["norm"] == "rms":
        x = x / (x.pow(2).mean(2, keepdim=True) + EPS).sqrt()
    x = x if weight is None else x * weight
    x = x if bias is None else x + bias
    axis = [k for k, n in enumerate(s["axes"]) for _ in range(n)]
    out = list(x.unbind(2))
    for j in range(half):
        i, k = (2 * j, 2 * j + 1) if c["interleaved"] else (j, half + j)
        z = torch.polar(torch.full((len(x), 1), s["amplitude"], dtype=F64, device="cuda"),
                        positions[:, axis[j], None].double() * f[j])
        w = torch.complex(x[..., i], x[..., k]) * z
        out[i], out[k] = w.real, w.imag
    return torch.stack(out, dim=2)


def _exact_back(name, s):
    names = [k for k in (name, name + "_weight", name + "_bias") if s[k] is not None]
    leaves = {k: s[k].double().contiguous().requires_grad_(True) for k in names}
    y = _exact_heads(leaves[name], leaves.get(name + "_weight"), leaves.get(name + "_bias"), s["positions"], s)
    grads = torch.autograd.grad((y.flatten(1) * s["d_" + name].double()).sum(), [leaves[k] for k in names])
    return dict(zip(names, (g.detach() for g in grads)))


def _exact_held(x):
    """The nearest values that blocks of 32 can hold, [rows, heads, head_dim]."""
    x = x.reshape(*x.shape[:2], -1, 32)
    power = torch.full(x.shape[:3], -120.0, dtype=F64, device="cuda")
    top = x.abs().amax(3)
    near = torch.where(top > 0, torch.log2(top.clamp(min=1e-300)).floor(), power)
    for e in (near - 3, near - 2, near - 1):  # the smallest power of two with no value above 7 times it
        power = torch.where((power == -120.0) & (top <= 7 * torch.exp2(e)), e.clamp(-120, 125), power)
    y = x * torch.exp2(-power)[..., None]
    grid = torch.tensor(GRID, dtype=F64, device="cuda")
    best, held = torch.full_like(y, math.inf), torch.zeros_like(y)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):  # the even codes first: they keep a tie
        off = (y.abs() - grid[code]).abs()
        held = torch.where(off < best, grid[code], held)
        best = torch.minimum(off, best)
    return (held * torch.sign(y) * torch.exp2(power)[..., None]).flatten(1)


def _exact_append4(s):
    c, start, before = s["c"], s["start"].tolist(), s["before"].tolist()
    rows, kept, positions = _rows(c), [], []
    for b in range(c["requests"]):
        m = start[b + 1] - start[b]
        for i in range(m):
            positions.append(c["first"] + before[b] + i)
            kept.append(not c["window"] or before[b] + i < c["sink"] or i >= m - c["window"])
    real = len(kept)
    kept = torch.tensor(kept + [False] * (rows - real), device="cuda")
    at = torch.tensor(positions + [0] * (rows - real), device="cuda")[:, None]
    at = at if s["positions"] is None else s["positions"]
    wide = {k: s[k].double() for k in ("q", "k", "v")}
    weight = {k: None if s[k] is None else s[k].double() for k in ("q_weight", "k_weight")}
    q = _exact_heads(wide["q"], weight["q_weight"], None, at, s).flatten(1)
    q[real:] = 0
    k = _exact_held(_exact_heads(wide["k"], weight["k_weight"], None, at, s))
    v = _exact_held(wide["v"].reshape(rows, -1, c["head_dim"]))
    return {"q": q, "k": k * kept[:, None], "v": v * kept[:, None]}


def _exact_attn4(s):
    c, start, lens = s["c"], s["start"].tolist(), s["lens"].tolist()
    d, g, p = c["head_dim"], c["heads"] // c["kv_heads"], c["page"]
    out, lse = s["out"].double(), s["lse"].double()
    value = torch.tensor([(-1) ** (i >> 3) * GRID[i & 7] for i in range(16)], dtype=F64, device="cuda")
    byte = torch.arange(256, device="cuda")
    pair = torch.stack((value[byte % 16], value[byte // 16]), dim=1)  # the two values of a byte

    def held(b, h, which):
        page = s["cache"][s["table"][b].long(), h]
        x = pair[page[:, which * p * d // 2:(which + 1) * p * d // 2].long()].reshape(-1, d // 32, 32)
        e = page[:, p * d:].reshape(-1, 2, d // 32)[:, which].double()
        return torch.ldexp(x, (e - 127)[..., None]).reshape(-1, d)[:lens[b]]

    for h in range(c["kv_heads"]):
        for b in range(c["requests"]):
            rows = slice(start[b], start[b + 1])
            if start[b] == start[b + 1]:
                continue
            k, v = held(b, h, 0), held(b, h, 1)
            for i in range(h * g, h * g + g):
                if not len(k):
                    out[rows, i * d:i * d + d], lse[i, rows] = 0, -math.inf
                    continue
                w = s["q"][rows, i * d:i * d + d].double() @ k.t().contiguous() / math.sqrt(d)
                lse[i, rows] = torch.logsumexp(w, 1)
                out[rows, i * d:i * d + d] = torch.softmax(w, 1) @ v
    return {"out": out, "lse": lse}


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "turn":
        w = {k: None if s[k] is None else s[k].double() for k in ("q_weight", "k_weight", "q_bias", "k_bias")}
        return {x: _exact_heads(s[x].double(), w[x + "_weight"], w[x + "_bias"], s["positions"], s).flatten(1)
                for x in ("q", "k")}
    if kind == "turn_grad":
        return {**_exact_back("q", s), **_exact_back("k", s)}
    return _exact_append4(s) if kind == "append4" else _exact_attn4(s)


# ------------------------------------------------------------------ work
def work(case):
    c = case
    d = c["head_dim"]
    hidden, kv = c["heads"] * d, c["kv_heads"] * d
    if c["kind"] in ("turn", "turn_grad"):
        n = c["rows"] * (hidden + kv)
        vectors = 8 * d * (c["weight"] + c["bias"])
        if c["kind"] == "turn":
            return {"bytes": 2 * n * SIZE[c["x"]] + 4 * c["rows"] * c["axes"] + vectors, "flops": 8 * n}
        return {"bytes": 3 * n * SIZE[c["x"]] + 4 * c["rows"] * c["axes"] + 2 * vectors, "flops": 16 * n}
    rows = c["requests"] * c["most"] / (1 if c["most"] == 1 else 2)  # the mean of the lengths
    if c["requests"] == 1:
        rows = c["most"]
    if c["kind"] == "append4":
        # q in and out; k and v in, into 4 bits and an exponent to 32, read and written out again
        held = 2 * kv * (0.5 + 1 / 32)
        return {"bytes": rows * (4 * hidden + 4 * kv + 2 * held + 4 * kv) + 20 * _rows(c), "flops": rows * 8 * (hidden + 2 * kv)}
    capacity = c["page"] * c["pages"]
    keys = capacity / 2 if c["requests"] > 1 else capacity - capacity // 4096
    return {"bytes": c["requests"] * keys * kv * 2 * (0.5 + 1 / 32) + rows * hidden * (2 + SIZE[c["out"]])
            + 4 * rows * c["heads"], "flops": 4 * rows * hidden * keys}
