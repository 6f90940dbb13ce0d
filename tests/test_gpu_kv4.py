"""The 4-bit cache on the GPU: the append against its definition in 64 bits (the numbers
themselves, without a tolerance: which one a key is rounded to is decided in 64 bits, and no
input here lies within 2^-40 of a border without lying on it), rows read back, attention over
it against softmax attention of the values that it holds.

Attention's tolerances. With w the exact weights, O = sum w_i v_i. The weights enter the
product as three bf16 parts for an fp32 output (24 bits: as they are), as two for a bf16 one
(2^-16 relative), or, for a bf16 output where more than 16 rows meet a key head, rounded to
bf16 (2^-8 relative) and normalised by the rounded sum, which moves O by
2^-8 sum w_i |v_i - O| <= 2^-8 (sum w_i |v_i| + |O|) at most. A score is an fp32 sum of head_dim exact products:
off by at most (head_dim + 8) 2^-24 max_i sum |q k_i| scale =: e, which moves a weight by 2 e
relative; 2^-20 covers the exponentials, the fp32 sums and the joins (each below 2^-22). So O is
off by (2^-16 (bf16) + 2 e + 2^-20) (sum w_i |v_i| + |O|), and its own rounding, |O| eps / 2; the LSE
by e + 2^-20 (1 + |LSE|). A weight below 2^-126 of the largest is below fp32's normal numbers
and may be lost, and so may the later parts (2^-8 at most) of one below 2^-117: less than
2^-120 sum |v_i| in all.
"""

import math

import pytest
import torch

import paper_2607_00712_amd as ispa
from kv4_format import decode, encode, pack, unpack
from test_gpu_norm_rotary import angles_of, check as check_turned, forward, pair_size, turn

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------ append and read
def exact_keys(k, w, b, p, f, axes, d, norm, interleaved, amplitude):
    """Keys [rows, heads, d] before they are rounded, in 64 bits."""
    if norm == "none":
        return turn(k.double().view(len(k), -1, d), angles_of(p, f, axes), interleaved, amplitude)
    return forward(k, w, b, p, f, axes, d, norm, interleaved, amplitude)[0].view(len(k), -1, d)


APPEND = [
    # counts, before, page, max_pages, window, heads, kv_heads, d, axes, interleaved, amplitude, norm, dtype, pad
    ([1], [0], 32, 1, 0, 1, 1, 64, (32,), True, 1.0, "none", BF16, 0),
    ([1] * 9, list(range(30, 39)), 32, 2, 0, 8, 2, 128, (64,), False, 1.25, "rms", BF16, 3),
    ([3, 0, 17, 1], [61, 5, 0, 127], 64, 2, 0, 6, 3, 64, (10, 6), False, 1.0, "layer", F32, 2),
    ([70, 33], [100, 0], 32, 6, 0, 12, 12, 128, (22, 21, 21), True, 1.0, "rms", BF16, 0),
    ([40, 300], [500, 20], 64, 2, 96, 4, 4, 64, (32,), True, 1.0, "none", BF16, 1),  # rings, more rows than their window
    ([2500], [0], 1024, 3, 0, 3, 1, 128, (64,), True, 1.0, "rms", BF16, 0),          # several tokens to a workgroup
    ([5, 6], [250, 3], 128, 2, 0, 2, 1, 128, (32,), False, 1.0, "rms", F32, 0),      # the last rows behind the capacity
    ([2, 2], [2, 9], 32, 1, 0, 32, 16, 64, (16,), True, 0.7, "layer", BF16, 0),
]


def append_case(case, seed=0):
    counts, before, page, pages, window, heads, kv, d, axes, _, _, norm, dtype, pad = APPEND[case]
    g = torch.Generator().manual_seed(17 * case + seed)
    r = lambda *s: torch.randn(*s, generator=g)
    rows = sum(counts) + pad
    start = torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32)
    n_pages = len(counts) * pages + 2
    t = dict(q=r(rows, heads * d).to(dtype), k=(r(rows, kv * d) * 1.5 + 0.2).to(dtype), v=r(rows, kv * d).to(dtype),
             start=start, before=torch.tensor(before, dtype=torch.int32), f=ispa.rotary_frequencies(axes, device="cpu")[0],
             p=torch.randint(0, 5000, (rows, len(axes)), generator=g, dtype=torch.int32),
             table=torch.randperm(n_pages, generator=g)[:len(counts) * pages].view(len(counts), pages).to(torch.int32),
             cache=torch.randint(0, 256, (n_pages, kv, page * (d + d // 16)), generator=g, dtype=torch.uint8))
    for n in ("q", "k"):
        t[n + "_weight"] = 1 + 0.3 * r(d) if norm != "none" else None
        t[n + "_bias"] = 0.2 * r(d) if norm == "layer" else None
    return t


def places(case, t, slots):
    """(page, row) of each row with a place, and which rows these are."""
    _, _, page, pages, *_ = APPEND[case]
    at = [(r, t["table"].view(-1)[s // page].item(), s % page) for r, s in enumerate(slots.tolist()) if s >= 0]
    return [(r, p, i) for r, p, i in at if 0 <= p < len(t["cache"])]


def append(case, t, **kw):
    counts, before, page, pages, window, heads, kv, d, axes, interleaved, amplitude, norm, dtype, pad = APPEND[case]
    g = {n: x.to(DEV) if isinstance(x, torch.Tensor) else x for n, x in t.items()}
    slots, _, _ = ispa.slot_map(g["start"], g["before"], page * pages, len(t["q"]),
                                sink=page * pages - window if window else 0, window=window)
    q = ispa.kv4_append(g["q"], g["k"], g["v"], g["p"], slots, g["f"], heads, g["cache"], g["table"], n_kv_heads=kv,
                        norm=norm, axes=axes, interleaved=interleaved, amplitude=amplitude,
                        **{n: g[n] for n in ("q_weight", "k_weight", "q_bias", "k_bias")}, **kw)
    return g, slots, q


@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(case):
    counts, before, page, pages, window, heads, kv, d, axes, interleaved, amplitude, norm, dtype, pad = APPEND[case]
    t = append_case(case)
    print(f"kv4_append {APPEND[case]}", flush=True)
    g, slots, q = append(case, t)
    torch.cuda.synchronize()
    keys = exact_keys(t["k"], t["k_weight"], t["k_bias"], t["p"], t["f"], axes, d, norm, interleaved, amplitude)
    values = t["v"].double().view(len(t["v"]), kv, d)
    want = [tuple(x.clone() for x in half) for half in unpack(t["cache"], d)]
    new = [encode(keys), encode(values)]
    at = places(case, t, slots.cpu())
    assert len(at) > 0
    for r, p, i in at:
        for (codes, powers), (c, e) in zip(want, new):
            codes[p, :, i], powers[p, :, i] = c[r], e[r]
    # every byte of the pool: the rows' places, and the others as they were (a negative zero is a zero)
    got = unpack(g["cache"].cpu(), d)
    for (gc, ge), (wc, we), what in zip(got, want, ("keys", "values")):
        assert torch.equal(ge, we), f"powers of the {what}"
        assert torch.equal(torch.where(gc == 8, 0, gc), torch.where(wc == 8, 0, wc)), f"codes of the {what}"
    # read back, with places that there are not
    k, v = ispa.kv4_read(g["cache"], g["table"], slots, d)
    k32, v32 = ispa.kv4_read(g["cache"], g["table"], slots, d, out_dtype=F32)
    held = {r for r, _, _ in at}
    for x, x32, (c, e) in ((k, k32, new[0]), (v, v32, new[1])):
        x, x32, y = x.cpu(), x32.cpu(), decode(c, e).flatten(1)
        y[[r for r in range(len(y)) if r not in held]] = 0
        assert torch.equal(x.double(), y) and torch.equal(x32.double(), y)
    # q, rounded once, as norm_rotary's tolerance has it
    if norm == "none":
        one = t["q"].double().view(len(t["q"]), -1, d)
        one, size = (x.flatten(1) for x in (turn(one, angles_of(t["p"], t["f"], axes), interleaved, amplitude),
                                            pair_size(one.abs(), len(t["f"]), interleaved, amplitude)))
    else:
        one, size = forward(t["q"], t["q_weight"], t["q_bias"], t["p"], t["f"], axes, d, norm, interleaved, amplitude)
    check_turned(q, one, size, 2.0 ** -19, "q")


@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_every_kind_of_append(d, dtype, norm):
    """Head sizes, types and norms, with and without weights and biases, part of a head turned."""
    rows, heads, kv, page = 37, 3, 5, 32
    g = torch.Generator().manual_seed(d + len(norm))
    r = lambda *s: torch.randn(*s, generator=g)
    f = ispa.rotary_frequencies(d // 4, device="cpu")[0]
    q, k, v = (r(rows, n * d).to(dtype) for n in (heads, kv, kv))
    p = torch.randint(0, 100000, (rows, 1), generator=g, dtype=torch.int32)
    put = lambda x: None if x is None else x.to(DEV)
    table, slots = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV), torch.arange(rows, device=DEV) + 9
    for weight, bias in [(False, False)] if norm == "none" else [(True, True), (True, False), (False, True), (False, False)]:
        vec = {n + what: (1 + 0.3 * r(d) if what == "_weight" else 0.2 * r(d)) if have else None
               for n in "qk" for what, have in (("_weight", weight), ("_bias", bias))}
        cache = ispa.kv4_cache(2, page, kv, d)
        out = ispa.kv4_append(put(q), put(k), put(v), put(p), slots, put(f), heads, cache, table, n_kv_heads=kv, norm=norm,
                              interleaved=bias, q_out=torch.empty(rows, heads * d, device=DEV),
                              **{n: put(x) for n, x in vec.items()})
        torch.cuda.synchronize()
        key, value = ispa.kv4_read(cache, table, slots, d, out_dtype=F32)
        exact_k = exact_keys(k, vec["k_weight"], vec["k_bias"], p, f, (d // 4,), d, norm, bias, 1.0)
        assert torch.equal(key.double().cpu(), decode(*encode(exact_k)).flatten(1))
        assert torch.equal(value.double().cpu(), decode(*encode(v.double().view(rows, kv, d))).flatten(1))
        if norm == "none":
            x = q.double().view(rows, heads, d)
            want, size = (x.flatten(1) for x in (turn(x, angles_of(p, f, (d // 4,)), bias, 1.0),
                                                 pair_size(x.abs(), d // 4, bias, 1.0)))
        else:
            want, size = forward(q, vec["q_weight"], vec["q_bias"], p, f, (d // 4,), d, norm, bias, 1.0)
        check_turned(out, want, size, 2.0 ** -19, "q")


def test_append_padding_and_places():
    """A given q_out keeps its padding; pages outside the pool and slots outside the table take
    nothing, and their rows' queries turn all the same; q in place in columns of one product."""
    case = 1
    t = append_case(case)
    heads, kv, d = 8, 2, 128
    _, _, plain = append(case, t)
    to = torch.full((len(t["q"]), heads * d), 9.0, dtype=BF16, device=DEV)
    g, slots, out = append(case, t, q_out=to, q_start=t["start"].to(DEV))
    real = int(t["start"][-1])
    assert out is to and torch.equal(out[:real], plain[:real]) and (out[real:] == 9).all()
    bad = dict(t, table=t["table"].clone())
    bad["table"][0], bad["table"][1] = -1, len(t["cache"])
    h, _, out = append(case, bad)
    assert torch.equal(out[:real], plain[:real])
    pages = [p for _, p, _ in places(case, bad, slots.cpu())]
    gone = sorted(set(range(len(t["cache"]))) - set(pages))
    assert torch.equal(h["cache"][gone].cpu(), t["cache"][gone])
    o = dict(n_kv_heads=kv, norm="rms", axes=(64,), interleaved=False, amplitude=1.25, q_weight=g["q_weight"],
             k_weight=g["k_weight"])
    far = torch.where(torch.arange(len(slots), device=DEV) % 2 == 0, slots, slots + (1 << 40))
    for s in (far, torch.full_like(slots, -(1 << 62))):
        cache = t["cache"].to(DEV)
        ispa.kv4_append(g["q"], g["k"], g["v"], g["p"], s, g["f"], heads, cache, g["table"], **o)
        keep = (s < 0) | (s >= 64 * 9)
        k, _ = ispa.kv4_read(cache, g["table"], s, d)
        assert (k[keep] == 0).all()
    assert torch.equal(cache, t["cache"].to(DEV))
    wide = torch.cat((g["q"], g["k"], g["v"]), 1)
    a, b, c = wide[:, :heads * d], wide[:, heads * d:heads * d + kv * d], wide[:, heads * d + kv * d:]
    cache = t["cache"].to(DEV)
    got = ispa.kv4_append(a, b, c, g["p"], slots, g["f"], heads, cache, g["table"], q_out=a, **o)
    assert torch.equal(got[:real], plain[:real]) and torch.equal(cache, g["cache"])
    assert torch.equal(b, g["k"]) and torch.equal(c, g["v"])


def test_every_rounding():
    """Borders, both sides of them, the ends of the range of powers, zeros, infinities and NaN,
    through values (as they are) and through keys at position zero."""
    d, rows = 64, 64
    g = torch.Generator().manual_seed(3)
    base = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, 7.0, 0.0, 0.1])
    x = torch.zeros(rows, d)
    for r in range(rows):
        power = 2.0 ** ((r * 7) % 60 - 30)
        y = base[torch.randint(0, 12, (d,), generator=g)] * (torch.randint(0, 2, (d,), generator=g) * 2 - 1)
        side = torch.randint(-1, 2, (d,), generator=g)
        y = torch.where(side == 0, y, torch.nextafter(y, y + side))
        x[r] = y * power
    x[1], x[2] = 0.0, x[2] * 0 + 1e-42
    x[3], x[4] = 3.3e38, -1e-36
    x[5, 3], x[6, 40], x[7, 63] = float("inf"), float("nan"), -float("inf")
    x[8] = torch.linspace(-7, 7, d)
    f = ispa.rotary_frequencies(32, device=DEV)[0]
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    slots = torch.arange(rows, device=DEV)
    cache = ispa.kv4_cache(2, 32, 1, d)
    one = x.to(DEV)
    q = ispa.kv4_append(one, one, one, torch.zeros(rows, dtype=torch.int32, device=DEV), slots, f, 1, cache, table)
    assert q.dtype == BF16
    want = encode(x.double())
    nan = torch.isnan(decode(*want))
    for got in ispa.kv4_read(cache, table, slots, d, out_dtype=F32):
        got = got.double().cpu()
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], decode(*want)[~nan])


def test_keys_on_their_side():
    """Keys normalised and turned far out, a quarter of a million of them: every number as 64
    bits decide."""
    rows, kv, d = 256, 8, 128
    g = torch.Generator().manual_seed(8)
    k = torch.randn(rows, kv * d, generator=g).to(BF16)
    w = 1 + 0.3 * torch.randn(d, generator=g)
    f, amplitude = ispa.rotary_frequencies(64, scaling="parts", factor=16.0, original_length=4096, device="cpu")
    p = torch.randint(900000, 1100000, (rows, 1), generator=g, dtype=torch.int32)
    cache, table = ispa.kv4_cache(8, 32, kv, d), torch.arange(8, dtype=torch.int32, device=DEV).view(1, 8)
    slots = torch.arange(rows, device=DEV)
    put = lambda x: x.to(DEV)
    ispa.kv4_append(put(k), put(k), put(k), put(p), slots, put(f), kv, cache, table, norm="rms", k_weight=put(w),
                    interleaved=False, amplitude=amplitude)
    got, _ = ispa.kv4_read(cache, table, slots, d)
    want = decode(*encode(exact_keys(k, w, None, p, f, (64,), d, "rms", False, amplitude))).flatten(1)
    assert torch.equal(got.double().cpu(), want)


# ------------------------------------------------------------------ attention
def make(counts, lens, page, pages, heads, kv_heads, d, pad=0, seed=0, q_scale=1.0):
    g = torch.Generator().manual_seed(seed + 13 * page + pages + len(counts))
    n = len(counts) * pages + 2
    r = lambda *s: torch.randn(*s, generator=g)
    rows = sum(counts) + pad
    k, v = encode(r(n, kv_heads, page, d)), encode(r(n, kv_heads, page, d) + 0.3)
    return dict(q=(r(rows, heads * d) * q_scale).to(BF16), cache=pack(k, v),
                table=torch.randperm(n, generator=g)[:len(counts) * pages].view(len(counts), pages).to(torch.int32),
                q_start=torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32),
                lens=torch.tensor(lens, dtype=torch.int32))


def on_gpu(t):
    return {k: v.to(DEV) for k, v in t.items()}


def exact(t, heads, scale=None):
    """out, lse, the tolerances of both (without the output's rounding) and sum w |v| + |O|."""
    rows, hidden = t["q"].shape
    d = hidden // heads
    scale = 1 / math.sqrt(d) if scale is None else scale
    (kc, ke), (vc, ve) = unpack(t["cache"], d)
    kv_heads, page = kc.shape[1:3]
    keys, values = decode(kc, ke), decode(vc, ve)
    out, tol, size = (torch.zeros(rows, hidden, dtype=torch.float64) for _ in range(3))
    lse = torch.full((heads, rows), -math.inf, dtype=torch.float64)
    lse_tol = torch.zeros(heads, rows, dtype=torch.float64)
    starts = t["q_start"].tolist()
    for b, length in enumerate(t["lens"].tolist()):
        at = slice(starts[b], starts[b + 1])
        n = min(max(length, 0), t["table"].shape[1] * page)
        place = torch.arange(n)
        pages = t["table"][b].long()[place // page]
        here = (pages >= 0) & (pages < len(keys))
        pages, row = pages[here], (place % page)[here]
        if not len(pages) or at.start == at.stop:
            continue
        for h in range(heads):
            c = h // (heads // kv_heads)
            kh, vh = keys[pages, c, row], values[pages, c, row]
            q = t["q"][at, h * d:(h + 1) * d].double()
            s = q @ kh.t() * scale
            w = torch.softmax(s, 1)
            o = w @ vh
            e = (d + 8) * 2.0 ** -24 * (q.abs() @ kh.abs().t()).amax(1) * abs(scale)
            out[at, h * d:(h + 1) * d] = o
            size[at, h * d:(h + 1) * d] = w @ vh.abs() + o.abs()
            tol[at, h * d:(h + 1) * d] = ((2 * e[:, None] + 2.0 ** -20) * size[at, h * d:(h + 1) * d]
                                          + 2.0 ** -120 * vh.abs().sum(0))
            lse[h, at] = torch.logsumexp(s, 1)
            lse_tol[h, at] = e + 2.0 ** -20 * (1 + lse[h, at].abs())
    return out, lse, tol, lse_tol, size


def check(got, got_lse, want, what="", rows=1):
    """rows: of a key head, as far as the call was told."""
    out, lse, tol, lse_tol, size = want
    if got.dtype == BF16:
        tol = tol + (2.0 ** -8 if rows > 16 else 2.0 ** -16) * size
    half = torch.finfo(got.dtype).eps / 2
    got, got_lse = got.double().cpu()[:len(out)], got_lse.double().cpu()
    full = torch.isfinite(lse)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    assert torch.equal(torch.isfinite(got_lse), full), f"{what}: lse"
    assert (got_lse[~full] == -math.inf).all(), f"{what}: lse of empty rows"
    over = (got - out).abs() - (tol + half * out.abs())
    assert torch.all(over <= 0), f"{what}: {over.max():.3e} over the tolerance"
    assert torch.all((got_lse - lse)[full].abs() <= lse_tol[full]), (
        f"{what}: lse {(got_lse - lse)[full].abs().max():.3e}")


@pytest.fixture(params=[0, 100])
def more(request):
    """Pages that there are not, behind the others: few pages and many take different ways."""
    return request.param


def attend(t, heads, more=0, **kw):
    table = torch.nn.functional.pad(t["table"], (0, more), value=-1)
    return ispa.attn_kv4(t["q"], t["cache"], table, t["q_start"], t["lens"], heads, **kw)


ATTN = [
    # counts, lens, page, pages, heads, kv_heads, d
    ([1], [0], 32, 1, 1, 1, 64), ([1], [1], 32, 1, 1, 1, 128), ([1, 1], [64, 0], 32, 2, 2, 2, 64),
    ([3, 0, 17, 1], [77, 5, 0, 33], 32, 3, 6, 2, 128), ([3, 0, 17, 1], [77, 5, 0, 33], 64, 2, 6, 2, 64),
    # keys that end around the units of 32 and the pages
    ([1, 2, 1, 3], [31, 32, 33, 1], 32, 2, 4, 4, 128), ([1, 2, 1, 3], [63, 64, 65, 0], 64, 2, 4, 4, 64),
    ([1, 2, 1, 3], [127, 128, 129, 96], 128, 2, 4, 1, 128), ([2, 2], [5, 200], 256, 1, 8, 8, 128),
    # items that lie in many runs, and runs that hold many items
    ([1] * 5, [3000, 0, 1, 2999, 512], 64, 47, 2, 2, 128), ([2], [7000], 1024, 7, 1, 1, 64), ([1], [9000], 32, 282, 1, 1, 128),
    ([1] * 300, [(37 * i) % 70 for i in range(300)], 32, 3, 4, 2, 64), ([2] * 40, [(31 * i) % 97 for i in range(40)], 32, 4, 8, 8, 128),
    # tiles of 16, 32 and 256 rows, and past them
    ([16], [40], 32, 2, 1, 1, 128), ([17], [40], 32, 2, 1, 1, 128), ([20, 20], [40, 64], 32, 2, 2, 2, 128),
    ([33], [300], 32, 10, 1, 1, 64), ([64], [90], 32, 3, 2, 1, 64), ([65], [300], 32, 10, 1, 1, 128),
    ([50, 50], [40, 700], 64, 11, 3, 1, 128), ([130, 70, 200], [300, 0, 701], 64, 11, 2, 2, 128),
    ([130, 70, 200], [300, 0, 701], 64, 11, 2, 1, 64), ([40, 1, 300], [33, 65, 129], 32, 5, 4, 2, 128),
    ([257, 3], [333, 50], 32, 11, 2, 2, 64), ([600], [1500], 512, 3, 2, 2, 128), ([513, 255, 256], [64, 65, 63], 64, 2, 2, 1, 128),
    # the largest shares of query heads to a key head
    ([1, 1, 1], [9, 8, 70], 32, 3, 64, 1, 64), ([5, 4], [9, 80], 32, 3, 48, 3, 128),
    # requests without rows around ones with rows
    ([0, 0, 2, 0], [5, 5, 5, 5], 32, 1, 2, 2, 128),
]


@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(case, out_dtype, more):
    counts, lens, page, pages, heads, kv_heads, d = ATTN[case]
    print(f"attn_kv4 {ATTN[case]} {out_dtype}", flush=True)
    t = make(counts, lens, page, pages, heads, kv_heads, d)
    g = on_gpu(t)
    out, lse = attend(g, heads, more, max_q=max(counts + [1]), out_dtype=out_dtype)
    again, lse2 = attend(g, heads, more, max_q=max(counts + [1]), out_dtype=out_dtype)
    torch.cuda.synchronize()
    check(out, lse, exact(t, heads), ATTN[case], max(counts) * heads // kv_heads)
    assert torch.equal(out, again) and torch.equal(lse, lse2)  # the same bits


@pytest.mark.parametrize("max_q", [1, 9, 20, 70, 5000])
@pytest.mark.parametrize("d", [64, 128])
def test_any_hint(max_q, d, more):
    """What the host knows of the rows changes the layout of the work alone."""
    t = make([1, 70, 0, 300, 9], [100, 33, 64, 257, 0], 64, 5, 2, 1, d, pad=4)
    g = on_gpu(t)
    out = torch.full_like(g["q"], 7.0)
    lse = torch.full((2, len(t["q"])), 7.0, device=DEV)
    attend(g, 2, more, max_q=max_q, out=out, lse=lse)
    torch.cuda.synchronize()
    assert (out[-4:] == 7).all() and (lse[:, -4:] == 7).all()  # padding is left as it was
    want = exact({**t, "q": t["q"][:-4]}, 2)
    check(out[:-4], lse[:, :-4], want, max_q, 2 * max_q)


@pytest.mark.parametrize("rows", [1, 20, 60, 300])
def test_keys_that_are_not_attended(rows, more):
    """What lies behind a request's end, in pages of no request, and pages that there are not:
    infinities and NaN there (power 255) change nothing."""
    t = make([rows, 2], [100, 37], 32, 5, 4, 2, 128)
    clean = attend(on_gpu(t), 4, more, max_q=rows)
    used = torch.zeros(len(t["cache"]), 32, dtype=torch.bool)
    for b, n in enumerate((100, 37)):
        for i in range(n):
            used[t["table"][b, i // 32], i % 32] = True
    (kc, ke), (vc, ve) = unpack(t["cache"], 128)
    spoil = lambda c, e: (torch.where(used[:, None, :, None], c, 15), torch.where(used[:, None, :, None], e, 255))
    spoilt = {**t, "cache": pack(spoil(kc, ke), spoil(vc, ve)), "table": t["table"].clone()}
    spoilt["table"][0, 4], spoilt["table"][1, 2:] = -7, 1 << 30
    got = attend(on_gpu(spoilt), 4, more, max_q=rows)
    assert all(torch.equal(a, b) for a, b in zip(got, clean))
    # pages out of the pool among the attended ones: as if their keys were not there
    holes = {**t, "table": t["table"].clone()}
    holes["table"][0, 1], holes["table"][1, 0] = -1, len(t["cache"])
    check(*attend(on_gpu(holes), 4, more, max_q=rows), exact(holes, 4), "holes", 2 * rows)
    holes["table"][:] = -1
    out, lse = attend(on_gpu(holes), 4, more, max_q=rows)
    assert (out == 0).all() and (lse == -math.inf).all()
    # a NaN that is attended shows in its rows alone
    bad = {**t, "cache": t["cache"].clone()}
    (_, e), _ = unpack(bad["cache"], 128)
    e[t["table"][1, 0], 1, 5, 2] = 255
    out, lse = attend(on_gpu(bad), 4, more, max_q=rows)
    assert torch.equal(out[:rows], clean[0][:rows]) and torch.isnan(lse[2:, rows:]).all()
    assert torch.equal(out[rows:, :256], clean[0][rows:, :256]) and torch.isnan(out[rows:, 256:]).all()


@pytest.mark.parametrize("q_scale", [8.0, 60.0])
@pytest.mark.parametrize("rows", [1, 30, 64, 290])
def test_large_scores(rows, q_scale, more):
    """Scores that grow along the keys, so that the softmax reference moves."""
    t = make([rows, 3], [700, 450], 64, 11, 2, 2, 128, q_scale=q_scale)
    (kc, ke), v = unpack(t["cache"], 128)
    for b in range(2):
        for i in range(11):  # later pages larger
            ke[t["table"][b, i]] += i // 3
    t["cache"] = pack((kc, ke), v)
    check(*attend(on_gpu(t), 2, more, max_q=rows, out_dtype=F32), exact(t, 2), q_scale)
    check(*attend(on_gpu(t), 2, more, max_q=rows, scale=0.01), exact(t, 2, 0.01), "scale", rows)


def test_every_value_shows(more):
    """One key of large weight in every place of a unit, and values of its own in every place:
    each output is that key's. The scores are whole numbers below 2^13, exact in fp32, and the
    largest is ahead by more than 1000, so that the other weights are zero: O = (hi + lo) v / w
    with hi + lo within 2^-16 w, a product and a division (2^-22): within 2^-15 |v|."""
    d, n = 128, 96
    k = torch.zeros(3, 1, 32, d, dtype=torch.float64)
    v = torch.zeros(3, 1, 32, d, dtype=torch.float64)
    g = torch.Generator().manual_seed(2)
    for i in range(n):
        sign = torch.randint(0, 2, (d,), generator=g) * 2.0 - 1
        k[i // 32, 0, i % 32] = 6 * sign
        v[i // 32, 0, i % 32] = NUM[torch.randint(0, 16, (d,), generator=g)] * 2.0 ** (i % 5)
    cache = pack(encode(k), encode(v))
    held = decode(*unpack(cache, d)[1])
    for rows in (1, 96):
        q = k.view(n, d)[:: n // rows].to(BF16)
        t = on_gpu(dict(q=q, cache=cache, table=torch.tensor([[0, 1, 2]], dtype=torch.int32),
                        q_start=torch.tensor([0, rows], dtype=torch.int32), lens=torch.tensor([n], dtype=torch.int32)))
        out, _ = attend(t, 1, more, scale=1.0, out_dtype=F32)
        want = held.view(n, d)[:: n // rows]
        assert torch.all((out.double().cpu() - want).abs() <= want.abs() * 2.0 ** -15)


NUM = torch.tensor([0.0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def test_layouts_streams_and_lengths_beyond():
    """q and out as columns of wider rows, another stream, lengths outside the capacity, pages
    that two requests share."""
    t = make([1, 5, 2], [200, 64, 3], 64, 3, 4, 4, 64)
    t["table"][1] = t["table"][0]
    g = on_gpu(t)
    want = attend(g, 4)
    wide = torch.zeros(8, 3 * 256, dtype=BF16, device=DEV)
    wide[:, 256:512] = g["q"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, lse = ispa.attn_kv4(wide[:, 256:512], g["cache"], g["table"], g["q_start"], g["lens"], 4, out=wide[:, :256])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want[0]) and torch.equal(lse, want[1]) and (wide[:, 512:] == 0).all()
    check(*want, exact(t, 4), "shared pages")
    t["lens"] = torch.tensor([2 ** 31 - 1, -5, 3], dtype=torch.int32)
    check(*attend(on_gpu(t), 4), exact(t, 4), "lengths")


@pytest.mark.parametrize("pages", [3, 40])
def test_starts_that_do_not_ascend(pages):
    """Request starts that go back name more rows than there are: nothing behind the workspace or
    the outputs is written."""
    n, rows, heads, d = 40, 50, 2, 64
    t = on_gpu(make([rows] + [0] * (n - 1), [70] * n, 32, pages, heads, 1, d))
    t["q_start"][1:n:2], t["q_start"][2:n:2] = rows, 0
    t["q_start"][n] = rows
    L = ispa.lib()
    need = L.ispa_attn_kv4_workspace_bytes(32, pages, n, rows, 1, heads, 1, d)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV)
    out = torch.full((rows + 8, heads * d), 3.0, dtype=BF16, device=DEV)
    st = L.ispa_attn_kv4(t["q"].data_ptr(), heads * d, t["cache"].data_ptr(), len(t["cache"]), 32, t["table"].data_ptr(), pages,
                         t["q_start"].data_ptr(), t["lens"].data_ptr(), n, rows, 1, heads, 1, d, 0.0, out.data_ptr(),
                         ispa.DTYPE_BF16, heads * d, None, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert st == ispa.ISPA_OK
    torch.cuda.synchronize()
    assert (ws[need:] == 77).all() and (out[rows:] == 3).all()


def test_many_requests():
    """More requests than a workgroup has threads, most of them without rows or keys, items and
    runs in every relation; tokens of every request as a call of its own."""
    n, d = 900, 64
    g = torch.Generator().manual_seed(6)
    counts = [(i * 7) % 3 if i % 5 else 0 for i in range(n)]
    lens = torch.randint(0, 64, (n,), generator=g).tolist()
    lens[450] = 32 * 64
    t = make(counts, lens, 32, 64, 2, 1, d)
    got = attend(on_gpu(t), 2, max_q=2, out_dtype=F32)
    check(*got, exact(t, 2), "many")
    for b in (3, 450, 899):
        at = slice(int(t["q_start"][b]), int(t["q_start"][b + 1]))
        one = dict(q=t["q"][at], cache=t["cache"], table=t["table"][b:b + 1].contiguous(),
                   q_start=torch.tensor([0, counts[b]], dtype=torch.int32), lens=t["lens"][b:b + 1])
        if counts[b]:
            check(*attend(on_gpu(one), 2, out_dtype=F32), exact(one, 2), b)


def test_rows_far_apart():
    """Rows of one wide tensor as far apart as they may be, over more than 2^32 elements: the same as
    rows side by side."""
    rows, heads, kv, d, ld = 260, 2, 1, 128, 1 << 24
    width = (heads + 2 * kv) * d
    wide = torch.empty((rows - 1) * ld + width, dtype=BF16, device=DEV)
    x = wide.as_strided((rows, width), (ld, 1))
    x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(3)).to(BF16))
    close = x.contiguous()
    f = ispa.rotary_frequencies(d // 2, device=DEV)[0]
    at, slots = torch.arange(rows, dtype=torch.int32, device=DEV), torch.arange(rows, device=DEV)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    start, lens = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([0, rows], [rows]))
    w = torch.linspace(0.5, 1.5, d, device=DEV)
    results = []
    for t in (x, close):
        q, k, v = t[:, :heads * d], t[:, heads * d:(heads + kv) * d], t[:, (heads + kv) * d:]
        cache = ispa.kv4_cache(2, 256, kv, d, device=DEV)
        turned = ispa.norm_rotary(q, k, at, f, heads, kv, q_weight=w)
        grads = ispa.norm_rotary_backward(q, k, q, k, at, f, heads, kv, q_weight=w)
        out = ispa.kv4_append(q, k, v, at, slots, f, heads, cache, table, kv, norm="rms", k_weight=w)
        seen = [y for n in (1, 20, rows) for y in ispa.attn_kv4(q, cache, table, start, lens, heads, max_q=n)]
        results.append([*turned, *grads.values(), out, cache, *seen])
    for i, (p, r) in enumerate(zip(*results)):
        assert torch.equal(p, r), i
    # outputs as far apart: in place, and attention's beside its queries
    q, k, v = x[:, :heads * d], x[:, heads * d:(heads + kv) * d], x[:, (heads + kv) * d:]
    ispa.norm_rotary(q, k, at, f, heads, kv, q_weight=w, q_out=q, k_out=k)
    assert torch.equal(q, results[1][0]) and torch.equal(k, results[1][1])
    ispa.attn_kv4(close[:, :d], cache, table, start, lens, 1, out=v)
    assert torch.equal(v, ispa.attn_kv4(close[:, :d], cache, table, start, lens, 1)[0])
    args = close[:, :heads * d], close[:, :d], close[:, :d], at, slots, f, heads, cache, table, kv
    ispa.kv4_append(*args, q_out=q)
    assert torch.equal(q, ispa.kv4_append(*args))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,pages", [(1, 1), (1, 8), (1, 48), (1, 49), (30, 7), (30, 47), (30, 49), (300, 2), (300, 24), (300, 25)])
def test_short_caches(rows, pages, d):
    """Capacities on both sides of where a workgroup takes an item whole, lengths from none to all, one
    request and several, and more items than the device has runs."""
    lens = [32 * pages, 0, 1, 16 * pages + 5, 32 * pages - 1, 31]
    several = [([rows], 2), ([rows, 2, rows, 1, 0, rows], 2), ([rows] * 6, 4 if rows < 300 else 1)]
    for counts, kv in several + [([3] * 700, 4)] * (pages == 1):
        t = make(counts, [lens[i % 6] for i in range(len(counts))], 32, pages, 4, kv, d)
        got = attend(on_gpu(t), 4, max_q=max(counts), out_dtype=F32)
        check(*got, exact(t, 4), f"{len(counts)} requests")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 20])
def test_items_of_many_runs(rows, d):
    """Items cut into some ten to thirty runs, which begin and end at every place of a workgroup's
    four: parts of runs, of whole workgroups, and of runs without any key (missing pages)."""
    for i, keys in enumerate([900, 1025, 1151, 1280, 1409, 1537, 1666, 1793, 2200, 2944, 3333, 4096]):
        t = make([rows, 1], [keys, 700], 32, 128, 4, 4, d, seed=i)
        if i % 3 == 1:
            t["table"][0, 5:22] = -1
        got = attend(on_gpu(t), 4, max_q=rows, out_dtype=F32)
        check(*got, exact(t, 4), keys)
        assert all(torch.equal(x, y) for x, y in zip(got, attend(on_gpu(t), 4, max_q=rows, out_dtype=F32)))


def test_far_pages():
    """A pool of more than 2^32 bytes: pages at its end are read, written and attended."""
    d, kv, page = 128, 8, 512
    n = (1 << 32) // (page * kv * (d + d // 16)) + 3
    cache = torch.empty(n, kv, page * (d + d // 16), dtype=torch.uint8, device=DEV)
    small = make([4], [700], page, 2, 8, kv, d)
    pages = torch.tensor([n - 1, n - 2], device=DEV)
    cache[pages] = small["cache"][small["table"][0].long()].to(DEV)
    t = on_gpu(small)
    far = dict(t, cache=cache, table=pages.to(torch.int32).view(1, 2))
    assert all(torch.equal(a, b) for a, b in zip(attend(far, 8), attend(t, 8)))
    slots = torch.tensor([0, 511, 512, 1023], device=DEV)
    assert all(torch.equal(a, b) for a, b in zip(ispa.kv4_read(cache, far["table"], slots, d),
                                                  ispa.kv4_read(t["cache"], t["table"], slots, d)))
    f = ispa.rotary_frequencies(64, device=DEV)[0]
    x, p = torch.randn(4, kv * d, device=DEV), torch.arange(4, dtype=torch.int32, device=DEV)
    for s in (far, t):
        ispa.kv4_append(x, x, x, p, slots, f, kv, s["cache"], s["table"])
    assert all(torch.equal(a, b) for a, b in zip(ispa.kv4_read(cache, far["table"], slots, d),
                                                  ispa.kv4_read(t["cache"], t["table"], slots, d)))


def test_graph():
    """Appends and attention of a step captured once and replayed: tokens, lengths and tables
    change between the replays, which eager work separates."""
    heads, kv, d, page, pages, n = 4, 2, 128, 32, 3, 3
    f = ispa.rotary_frequencies(64, device=DEV)[0]
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g).to(BF16).to(DEV)
    q, k, v = r(n, heads * d), r(n, kv * d), r(n, kv * d)
    start = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    before = torch.tensor([0, 31, 60], dtype=torch.int32, device=DEV)
    table = torch.arange(n * pages, dtype=torch.int32, device=DEV).view(n, pages)
    caches = [ispa.kv4_cache(n * pages, page, kv, d) for _ in range(2)]

    def step(cache):
        slots, positions, lens = ispa.slot_map(start, before, page * pages, n)
        turned = ispa.kv4_append(q, k, v, positions, slots, f, heads, cache, table, n_kv_heads=kv, norm="rms")
        return ispa.attn_kv4(turned, cache, table, start, lens, heads, max_q=1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[0])
    torch.cuda.current_stream().wait_stream(side)
    step(caches[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(caches[0])
    for i in range(4):
        q.copy_(r(n, heads * d))
        k.copy_(r(n, kv * d))
        before.add_(1)
        if i == 2:
            table.copy_(table.flip(0).clone())
        graph.replay()
        want = step(caches[1])
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(*caches)


def test_step_of_a_layer():
    """A stream's chunks as they are used: norm, rotation and append of each chunk, attention over
    all of them, and the history's rows handed to a bf16 cache, whose chunk attention agrees."""
    heads, d, chunk, page = 2, 64, 70, 64
    f = ispa.rotary_frequencies((12, 10, 10), device=DEV)[0]
    g = torch.Generator().manual_seed(4)
    cache, table = ispa.kv4_cache(5, page, heads, d), torch.tensor([[3, 0, 4, 1]], dtype=torch.int32, device=DEV)
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(DEV)
    start = torch.tensor([0, chunk], dtype=torch.int32, device=DEV)
    lens = torch.zeros(1, dtype=torch.int32, device=DEV)
    for i in range(3):
        wide = torch.randn(chunk, 3 * heads * d, generator=g).to(BF16).to(DEV)
        q, k, v = wide.chunk(3, dim=1)
        slots, _, lens = ispa.slot_map(start, lens, 4 * page, chunk)
        at = torch.stack((torch.full((chunk,), i), torch.arange(chunk) // 10, torch.arange(chunk) % 10), 1).int().to(DEV)
        turned = ispa.kv4_append(q, k, v, at, slots, f, heads, cache, table, norm="rms", q_weight=w, k_weight=w,
                                 axes=(12, 10, 10))
        out, lse = ispa.attn_kv4(turned, cache, table, start, lens, heads, out_dtype=F32)
    n = 3 * chunk
    assert lens.item() == n
    k, v = ispa.kv4_read(cache, table, torch.arange(n, device=DEV), d)
    same, lse2 = ispa.attn_chunk(turned, k, v, n, n, heads)
    # chunk attention rounds its weights to bf16: 2^-8 (sum w |v| + |O|)
    t = dict(q=turned.cpu(), cache=cache.cpu(), table=table.cpu(), q_start=start.cpu(), lens=lens.cpu())
    want = exact(t, heads)
    check(out, lse, want, "4-bit", chunk)
    assert torch.all((same.double().cpu() - want[0]).abs() <= want[2] + 2.0 ** -8 * want[4])
    assert torch.all((lse2 - lse).abs().double().cpu() <= 2 * want[3])
    local = ispa.LocalKV(k, v, n, 64, 16)
    assert local.rows == 80 and torch.equal(local.k[16:], k[n - 64:])


def test_refusals():
    t = on_gpu(make([2, 1], [40, 3], 32, 2, 4, 2, 64))
    ok = lambda **kw: ispa.attn_kv4(**{**dict(q=t["q"], cache=t["cache"], page_table=t["table"], q_start=t["q_start"],
                                             cache_lens=t["lens"], n_heads=4), **kw})
    ok()
    assert ok(q=t["q"][:0])[0].shape == (0, 256)
    for error, kw in [(TypeError, dict(q=t["q"].float())), (ValueError, dict(n_heads=3)), (ValueError, dict(n_heads=1)),
                      (TypeError, dict(cache=t["cache"].float())), (ValueError, dict(cache=t["cache"][:, :, :-1])),
                      (ValueError, dict(page_table=t["table"][:1])), (TypeError, dict(page_table=t["table"].long())),
                      (ValueError, dict(q_start=t["q_start"][:2])), (ValueError, dict(cache_lens=t["lens"][:1])),
                      (ValueError, dict(out=t["q"][:2].clone())), (ispa.IspaError, dict(out=t["q"])),
                      (ispa.IspaError, dict(max_q=0)), (ValueError, dict(cache_lens=t["lens"].cpu()))]:
        with pytest.raises(error):
            ok(**kw)
    f = ispa.rotary_frequencies(32, device=DEV)[0]
    k = t["q"][:, :128].contiguous()
    p, slots = torch.zeros(3, dtype=torch.int32, device=DEV), torch.arange(3, device=DEV)
    ok = lambda **kw: ispa.kv4_append(**{**dict(q=t["q"], k=k, v=k, positions=p, slots=slots, freqs=f, n_heads=4,
                                               n_kv_heads=2, cache=t["cache"], page_table=t["table"]), **kw})
    ok()
    for error, kw in [(ValueError, dict(norm="batch")), (ispa.IspaError, dict(q_weight=torch.ones(64, device=DEV))),
                      (ValueError, dict(n_kv_heads=1)), (TypeError, dict(slots=slots.int())), (ValueError, dict(v=k[:2])),
                      (ValueError, dict(slots=slots[:2])), (ValueError, dict(q_start=t["q_start"][:2])),
                      (ispa.IspaError, dict(q_out=t["q"][:, :].view(3, 256)[:, :], k=t["q"][:, :128])),
                      (TypeError, dict(v=k.float()))]:
        with pytest.raises(error):
            ok(**kw)
    with pytest.raises(ispa.IspaError):
        ispa.kv4_cache(4, 48, 1, 64)
    with pytest.raises(ispa.IspaError):  # pages of 16 tokens of 128 values
        ispa.kv4_read(t["cache"], t["table"], slots, 128)
