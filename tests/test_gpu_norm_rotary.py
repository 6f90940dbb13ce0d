"""norm_rotary and its backward pass on the GPU against their definitions in 64 bits.

u = 2^-24. Forward: the deviation's sum of squares goes through at most 16 + 4 additions
of positive terms, a root and a division (below 15 u in all for the reciprocal deviation);
n w takes two more roundings and b one: n w + b is off by 18 u (|n w| + |b|), and with a
mean by 24 u of mean|x| r |w| more; cos and sin by 2^-21 (|a| + |b|) of the pair. Together
below 2^-19 of the pair's |n w| + |b| + mean|x| r |w|, times the amplitude, and the output's
own rounding, |value| eps / 2.

Backward: du is off by 8 u of its pair, n by 18 u of N = |n| + mean|x| r, the means of g and
of g n (sums of head_dim terms) by 22 u more, r by 15 u: dx by less than 2^-17 of
r (G + mean G + N mean(G N)) with G the pair's |dz| amplitude |w|. A sum over rows and heads
runs over a thread's heads, up to 256 threads and 128 + 8 workgroups (below 600 additions at
these sizes, with each term's own error below 2^-14) of |du| N or |du|.
"""

import pytest
import torch

import paper_2607_00712_amd as ispa

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


def pairs_of(t, half, interleaved):
    j = torch.arange(half)
    i, k = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
    return t[..., i], t[..., k], i, k


def turn(x, angles, interleaved, amplitude, sign=1):
    """x [rows, heads, d] turned, and the magnitudes of each value's pair."""
    c, s = (angles.cos() * amplitude)[:, None], (angles.sin() * amplitude * sign)[:, None]
    a, b, i, k = pairs_of(x, angles.shape[1], interleaved)
    out = x.clone()
    out[..., i], out[..., k] = a * c - b * s, a * s + b * c
    return out


def pair_size(x, half, interleaved, amplitude):
    a, b, i, k = pairs_of(x, half, interleaved)
    out = x.clone()
    out[..., i] = out[..., k] = (a + b) * abs(amplitude)
    return out


def normed(x, norm):
    mean = x.mean(-1, keepdim=True) if norm == "layer" else torch.zeros_like(x[..., :1])
    r = 1 / ((x - mean).square().mean(-1, keepdim=True) + EPS).sqrt()
    n = (x - mean) * r
    spread = x.abs().mean(-1, keepdim=True) * r if norm == "layer" else torch.zeros_like(r)
    return n, r, spread


def angles_of(p, f, axes):
    axis = torch.tensor([k for k, n in enumerate(axes) for _ in range(n)])
    return p.double().view(len(p), -1)[:, axis] * f


def forward(x, w, b, p, f, axes, d, norm, interleaved, amplitude):
    x = x.double().view(len(x), -1, d)
    n, _, spread = normed(x, norm)
    w = torch.ones(d, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(d, dtype=torch.float64) if b is None else b.double()
    out = turn(n * w + b, angles_of(p, f, axes), interleaved, amplitude)
    size = pair_size((n * w).abs() + b.abs() + spread * w.abs(), len(f), interleaved, amplitude)
    return out.flatten(1), size.flatten(1)


def backward(dz, x, w, p, f, axes, d, norm, interleaved, amplitude):
    """dx, dw, db and the magnitudes of each."""
    x, dz = x.double().view(len(x), -1, d), dz.double().view(len(x), -1, d)
    n, r, spread = normed(x, norm)
    w = torch.ones(d, dtype=torch.float64) if w is None else w.double()
    du = turn(dz, angles_of(p, f, axes), interleaved, amplitude, -1)
    size = pair_size(dz.abs(), len(f), interleaved, amplitude)
    g, N = du * w, n.abs() + spread
    m = g.mean(-1, keepdim=True) if norm == "layer" else 0
    dx = r * (g - m - n * (g * n).mean(-1, keepdim=True))
    G = size * w.abs()
    dx_size = r * (G + G.mean(-1, keepdim=True) + N * (G * N).mean(-1, keepdim=True))
    return ((dx.flatten(1), dx_size.flatten(1)), ((du * n).sum((0, 1)), (size * N).sum((0, 1))),
            (du.sum((0, 1)), size.sum((0, 1))))


def check(got, want, size, share, what):
    got = got.cpu()
    tol = want.abs() * (torch.finfo(got.dtype).eps / 2) + size * share
    over = (got.double() - want).abs() - tol
    assert torch.isfinite(got).all() and torch.all(over <= 0), f"{what}: {over.max().item():.3e} over the tolerance"


CASES = [
    # rows, heads, kv_heads, head_dim, axes, interleaved, amplitude, norm, weight, bias, dtype, far
    (1, 1, 1, 16, (8,), True, 1.0, "rms", True, True, F32, 1),
    (3, 2, 1, 64, (32,), False, 1.2, "layer", True, False, BF16, 1),
    (5, 3, 3, 64, (16,), False, 1.0, "rms", False, True, F32, 1),
    (7, 12, 12, 128, (22, 21, 21), True, 1.0, "rms", True, False, BF16, 1),
    (64, 32, 8, 128, (64,), False, 1.25, "rms", True, False, BF16, 1000003),
    (33, 5, 2, 48, (8, 16), True, 0.5, "layer", True, True, F32, 1),
    (29, 9, 3, 96, (24,), False, 1.0, "layer", True, True, F32, 1),
    (13, 4, 2, 80, (40,), True, 1.0, "rms", True, False, BF16, 1),
    (2, 10, 2, 256, (32, 32, 32, 32), False, 1.0, "layer", False, False, BF16, 1),
    (2050, 2, 1, 64, (32,), True, 1.0, "rms", True, True, BF16, 1),
    (8201, 1, 1, 32, (16,), False, 1.0, "rms", True, False, F32, 2 ** 31 - 40),
    (4, 300, 1, 64, (32,), True, 1.0, "layer", True, False, F32, -5000),
]


def inputs(case, seed=0):
    rows, heads, kv, d, axes, _, _, _, weight, bias, dtype, far = CASES[case]
    g = torch.Generator().manual_seed(rows + heads + seed)
    r = lambda *s: torch.randn(*s, generator=g)
    p = torch.randint(0, 37, (rows, len(axes)), generator=g, dtype=torch.int32)
    p += (torch.randint(0, 3, (rows, len(axes)), generator=g, dtype=torch.int32) * (far // 3)) if far != 1 else 0
    f, _ = ispa.rotary_frequencies(axes, device="cpu")
    t = dict(q=(r(rows, heads * d) + 0.5).to(dtype), k=(r(rows, kv * d) * 2).to(dtype), d_q=r(rows, heads * d).to(dtype),
             d_k=r(rows, kv * d).to(dtype), p=p, f=f)
    for x in ("q", "k"):
        t[x + "_weight"] = 1 + 0.3 * r(d) if weight else None
        t[x + "_bias"] = 0.2 * r(d) if bias else None
    return t


def options(case, t, device=DEV):
    _, _, kv, _, axes, interleaved, amplitude, norm, _, _, _, _ = CASES[case]
    put = lambda x: None if x is None else x.to(device)
    return dict(n_kv_heads=kv, norm=norm, eps=EPS, axes=axes, interleaved=interleaved, amplitude=amplitude,
                **{n: put(t[n]) for n in ("q_weight", "k_weight", "q_bias", "k_bias")})


@pytest.mark.parametrize("out_dtype", [None, BF16, F32])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward(case, out_dtype):
    rows, heads, kv, d, axes, interleaved, amplitude, norm, *_ = CASES[case]
    t = inputs(case)
    print(f"norm_rotary {CASES[case]} {out_dtype}", flush=True)
    got = ispa.norm_rotary(t["q"].to(DEV), t["k"].to(DEV), t["p"].to(DEV), t["f"].to(DEV), heads, out_dtype=out_dtype,
                           **options(case, t))
    torch.cuda.synchronize()
    for name, x in zip("qk", got):
        assert x.dtype == (out_dtype or t["q"].dtype)
        want, size = forward(t[name], t[name + "_weight"], t[name + "_bias"], t["p"], t["f"], axes, d, norm, interleaved,
                             amplitude)
        check(x, want, size, 2.0 ** -19, name)


@pytest.mark.parametrize("case", range(len(CASES)))
def test_backward(case):
    rows, heads, kv, d, axes, interleaved, amplitude, norm, *_ = CASES[case]
    t = inputs(case)
    print(f"norm_rotary_backward {CASES[case]}", flush=True)
    args = [t[n].to(DEV) for n in ("d_q", "d_k", "q", "k", "p", "f")]
    got = ispa.norm_rotary_backward(*args, heads, **options(case, t))
    again = ispa.norm_rotary_backward(*args, heads, **options(case, t))
    torch.cuda.synchronize()
    assert got.keys() == again.keys() and all(torch.equal(got[n], again[n]) for n in got)  # the same bits
    for name in "qk":
        (dx, dx_size), (dw, dw_size), (db, db_size) = backward(t["d_" + name], t[name], t[name + "_weight"], t["p"],
                                                               t["f"], axes, d, norm, interleaved, amplitude)
        check(got[name], dx, dx_size, 2.0 ** -17, name)
        for n, want, size in ((name + "_weight", dw, dw_size), (name + "_bias", db, db_size)):
            assert (n in got) == (t[n] is not None)
            if n in got:
                check(got[n], want, size, 2.0 ** -14, n)


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("types", [(BF16, F32), (F32, BF16), (BF16, BF16), (F32, F32)])
def test_every_kind_of_gradient(types, bias, norm):
    """Types of the values and of the gradients, with and without a bias's."""
    rows, heads, kv, d, axes = 53, 7, 2, 128, (40, 24)
    g = torch.Generator().manual_seed(11)
    r = lambda *s: torch.randn(*s, generator=g)
    x = {"q": (r(rows, heads * d) + 0.3).to(types[0]), "k": r(rows, kv * d).to(types[0])}
    dz = {"q": r(rows, heads * d).to(types[1]), "k": r(rows, kv * d).to(types[1])}
    w = {n: 1 + 0.3 * r(d) for n in "qk"}
    p = torch.randint(0, 5000, (rows, 2), generator=g, dtype=torch.int32)
    f, _ = ispa.rotary_frequencies(axes, device="cpu")
    b = torch.zeros(d, device=DEV) if bias else None
    put = lambda t: t.to(DEV)
    got = ispa.norm_rotary_backward(put(dz["q"]), put(dz["k"]), put(x["q"]), put(x["k"]), put(p), put(f), heads, kv, norm,
                                    put(w["q"]), put(w["k"]), b, b, axes=axes, interleaved=bias, amplitude=0.8)
    torch.cuda.synchronize()
    for n in "qk":
        (dx, dx_size), (dw, dw_size), (db, db_size) = backward(dz[n], x[n], w[n], p, f, axes, d, norm, bias, 0.8)
        assert got[n].dtype == types[0]
        check(got[n], dx, dx_size, 2.0 ** -17, n)
        check(got[n + "_weight"], dw, dw_size, 2.0 ** -14, n + "_weight")
        if bias:
            check(got[n + "_bias"], db, db_size, 2.0 ** -14, n + "_bias")


def test_gradient_against_differences():
    """<gradient, direction> against differences of the definition: steps h and 2 h, whose
    disagreement is three times the error of the smaller one."""
    case = 5
    rows, heads, kv, d, axes, interleaved, amplitude, norm, *_ = CASES[case]
    t = inputs(case)
    got = ispa.norm_rotary_backward(*[t[n].to(DEV) for n in ("d_q", "d_k", "q", "k", "p", "f")], heads,
                                    **options(case, t))
    g = torch.Generator().manual_seed(5)
    for name in "qk":
        leaves = {n: t[n].double() for n in (name, name + "_weight", name + "_bias")}
        step = {n: torch.randn(x.shape, generator=g, dtype=torch.float64) for n, x in leaves.items()}

        def f(h):
            x, w, b = (leaves[n] + h * step[n] for n in leaves)
            return (forward(x, w, b, t["p"], t["f"], axes, d, norm, interleaved, amplitude)[0] * t["d_" + name].double()).sum()

        one, two = ((f(h) - f(-h)) / (2 * h) for h in (1e-4, 2e-4))
        mine = sum((got[n].double().cpu() * step[n]).sum() for n in leaves)
        # the gradients' own tolerances, met by the direction
        sizes = backward(t["d_" + name], t[name], t[name + "_weight"], t["p"], t["f"], axes, d, norm, interleaved,
                         amplitude)
        own = sum(((s * c + w.abs() * 2.0 ** -24) * step[n].abs()).sum()
                  for (w, s), c, n in zip(sizes, (2.0 ** -17, 2.0 ** -14, 2.0 ** -14), leaves))
        assert abs(mine - one) <= own + abs(one - two) + 1e-9 * abs(one)


@pytest.mark.parametrize("place", ["in place", "one product", "apart", "q alone"])
def test_layouts(place):
    """q and k turned in place, as columns of one product, into columns of another tensor, and
    q alone: the same bits as separate tensors."""
    case = 4
    rows, heads, kv, d, *_ = CASES[case]
    t = inputs(case)
    q, k, p, f = (t[n].to(DEV) for n in ("q", "k", "p", "f"))
    o = options(case, t)
    want = ispa.norm_rotary(q, k, p, f, heads, **o)
    if place == "q alone":
        o = {n: x for n, x in o.items() if not n.startswith("k_")}
        got, none = ispa.norm_rotary(q, None, p, f, heads, **o)
        assert none is None and torch.equal(got, want[0])
        d_q = t["d_q"].to(DEV)
        one = ispa.norm_rotary_backward(d_q, None, q, None, p, f, heads, **o)
        two = ispa.norm_rotary_backward(d_q, t["d_k"].to(DEV), q, k, p, f, heads, **options(case, t))
        assert set(one) == {"q", "q_weight"} and all(torch.equal(one[n], two[n]) for n in one)
        return
    wide = torch.cat((q, k, torch.full((rows, 40), 7.0, dtype=BF16, device=DEV)), 1)
    rest = wide[:, -40:].clone()
    a, b = wide[:, :heads * d], wide[:, heads * d:(heads + kv) * d]
    if place == "in place":
        got = ispa.norm_rotary(q, k, p, f, heads, q_out=q, k_out=k, **o)
    elif place == "one product":
        got = ispa.norm_rotary(a, b, p, f, heads, q_out=a, k_out=b, **o)
    else:
        to = torch.full((rows, (heads + kv) * d + 8), 3.0, dtype=BF16, device=DEV)
        got = ispa.norm_rotary(a, b, p, f, heads, q_out=to[:, kv * d:kv * d + heads * d], k_out=to[:, :kv * d], **o)
        assert torch.equal(to[:, -8:], torch.full((rows, 8), 3.0, dtype=BF16, device=DEV))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(wide[:, -40:], rest)
    # the gradient reads such columns too
    if place == "apart":
        wide_d = torch.cat((t["d_k"], t["d_q"]), 1).to(DEV)
        one = ispa.norm_rotary_backward(wide_d[:, kv * d:], wide_d[:, :kv * d], a, b, p, f, heads, **o)
        two = ispa.norm_rotary_backward(t["d_q"].to(DEV), t["d_k"].to(DEV), q, k, p, f, heads, **o)
        assert all(torch.equal(one[n], two[n]) for n in two)


def test_special_values():
    """Zero rows give the bias turned; an infinity or a NaN spoils its own head alone."""
    d, heads = 64, 3
    p = torch.zeros(2, dtype=torch.int32, device=DEV)
    f, _ = ispa.rotary_frequencies(32, device=DEV)
    bias = torch.linspace(-1, 1, d, device=DEV)
    x = torch.randn(2, heads * d, device=DEV)
    clean, _ = ispa.norm_rotary(x, None, p, f, heads, q_bias=bias)
    bad = x.clone()
    bad[0, :d] = 0
    bad[1, d + 5] = float("inf")
    bad[1, 2 * d] = float("nan")
    got, _ = ispa.norm_rotary(bad, None, p, f, heads, q_bias=bias)
    assert torch.equal(got[0, :d], bias) and torch.equal(got[0, d:], clean[0, d:]) and torch.equal(got[1, :d], clean[1, :d])
    assert not torch.isfinite(got[1, d:2 * d]).all() and torch.isnan(got[1, 2 * d:]).all()


def test_empty_and_graph():
    """No rows; and a step (forward and backward) captured and replayed over changing inputs,
    with eager work between the replays."""
    case = 3
    rows, heads, kv, d, *_ = CASES[case]
    t = inputs(case)
    o = options(case, t)
    q, k, p, f, d_q, d_k = (t[n].to(DEV) for n in ("q", "k", "p", "f", "d_q", "d_k"))
    none = ispa.norm_rotary(q[:0], k[:0], p[:0], f, heads, **o)
    assert none[0].shape == (0, heads * d)
    back = ispa.norm_rotary_backward(d_q[:0], d_k[:0], q[:0], k[:0], p[:0], f, heads, **o)
    assert back["q_weight"].eq(0).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ispa.norm_rotary(q, k, p, f, heads, **o)
        ispa.norm_rotary_backward(d_q, d_k, q, k, p, f, heads, **o)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ispa.norm_rotary(q, k, p, f, heads, **o)
        grads = ispa.norm_rotary_backward(d_q, d_k, q, k, p, f, heads, **o)
    for i in range(3):
        n = inputs(case, seed=i)
        q.copy_(n["q"])
        d_k.copy_(n["d_k"])
        graph.replay()
        want = ispa.norm_rotary(q, k, p, f, heads, **o)
        want_g = ispa.norm_rotary_backward(d_q, d_k, q, k, p, f, heads, **o)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and all(torch.equal(grads[x], want_g[x]) for x in want_g)


def test_refusals():
    q = torch.zeros(4, 256, dtype=BF16, device=DEV)
    p, w = torch.zeros(4, dtype=torch.int32, device=DEV), torch.ones(64, device=DEV)
    f, _ = ispa.rotary_frequencies(32, device=DEV)
    ok = lambda **kw: ispa.norm_rotary(**{**dict(q=q, k=q[:, :64].contiguous(), positions=p, freqs=f, n_heads=4,
                                                 n_kv_heads=1), **kw})
    ok()
    for error, kw in [(ValueError, dict(norm="none")), (ValueError, dict(n_heads=3)), (ValueError, dict(k_weight=w, k=None)),
                      (ValueError, dict(q_weight=w[:32])), (TypeError, dict(q_weight=w.double())),
                      (TypeError, dict(q=q.half())), (TypeError, dict(k=q[:, :64].float())),
                      (ValueError, dict(k=q[:3, :64])), (ValueError, dict(n_kv_heads=2)),
                      (ValueError, dict(q_out=q[:3])), (TypeError, dict(q_out=q.float(), k_out=q[:, :64].clone())),
                      (ValueError, dict(positions=p[:3])), (ValueError, dict(q=q.cpu())),
                      (ispa.IspaError, dict(q_out=q[:, :], k_out=q[:, :64])), (ispa.IspaError, dict(eps=-1.0))]:
        with pytest.raises(error):
            ok(**kw)
