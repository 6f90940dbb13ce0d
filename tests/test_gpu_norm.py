"""norm_residual and its backward pass on the GPU against their formulas in 64 bits.

Tolerances. An output rounds once: |value| eps(dtype) / 2. Before that everything is
fp32: a row's sum passes at most 32 values a lane, 6 steps over lanes and 16 waves, so
that with the few roundings around it every quantity is within 64 x 2^-24 = 2^-18 of
the sum of the magnitudes that enter it (`size` below). A vector's gradient passes at
most the rows of a workgroup, its slots and the workgroups' slices in turn: fewer than
256 additions at these sizes, 2^-16 of the sum of the magnitudes, and each term carries
its own 2^-18.
"""

import pytest
import torch

import paper_2607_00712_amd as ispa

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
ROW, COL = 2.0 ** -18, 2.0 ** -16


def half_step(t):
    return torch.finfo(t).eps / 2


def make(rows, cols, x=F32, y=BF16, h=BF16, norm="layer", weight=False, bias=False, scale=False, shift=False,
         post="none", post_weight=False, gate=False, group=None, seed=0):
    g = torch.Generator().manual_seed(seed + 7 * rows + cols)
    r = lambda *s: torch.randn(*s, generator=g)
    groups = -(-rows // group) if group else 1
    c = dict(norm=norm, post=post, alpha=0.75, group_rows=group, eps=1e-6)
    t = dict(x=(r(rows, cols) * torch.exp(2 * r(rows, 1)) + r(1, cols)).to(x))
    t["y"] = (r(rows, cols) + 0.5).to(y) if y is not None else None
    for name, on, shape in (("weight", weight, (cols,)), ("bias", bias, (cols,)), ("scale", scale, (groups, cols)),
                            ("shift", shift, (groups, cols)), ("post_weight", post_weight, (cols,)),
                            ("gate", gate, (groups, cols))):
        t[name] = r(*shape) if on else None
    return c, t, h


def wide(t, grad=False):
    out = {k: None if v is None else v.double().requires_grad_(grad) for k, v in t.items()}
    return out


def spread(v, c, rows):
    return v.repeat_interleave(c["group_rows"] or max(rows, 1), dim=0)[:rows]


def normed(x, kind, eps):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    return x / (x.pow(2).mean(1, keepdim=True) + eps).sqrt()


def stream(c, t):
    if t["y"] is None:
        return t["x"]
    z = normed(t["y"], c["post"], c["eps"])
    z = z if t["post_weight"] is None else z * t["post_weight"]
    z = z if t["gate"] is None else z * spread(t["gate"], c, len(z))
    return t["x"] + c["alpha"] * z


def head(c, t, x):
    h = normed(x, c["norm"], c["eps"])
    h = h if t["weight"] is None else h * t["weight"]
    h = h if t["bias"] is None else h + t["bias"]
    h = h if t["scale"] is None else h * (1 + spread(t["scale"], c, len(h)))
    return h if t["shift"] is None else h + spread(t["shift"], c, len(h))


def size_of_norm(x, kind, eps):
    """The magnitudes that enter a normalised value."""
    if kind == "none":
        return x.abs()
    rms = x.pow(2).mean(1, keepdim=True).sqrt()
    dev = x - x.mean(1, keepdim=True) if kind == "layer" else x
    return (x.abs() + rms) / (dev.pow(2).mean(1, keepdim=True) + eps).sqrt() + dev.abs() / (
        dev.pow(2).mean(1, keepdim=True) + eps).sqrt()


def sizes(c, t, x):
    """The magnitudes that enter x_out and h."""
    one = {k: None if v is None else v.abs() for k, v in t.items()}
    sx = t["x"].abs()
    if t["y"] is not None:
        z = size_of_norm(t["y"], c["post"], c["eps"])
        z = z if one["post_weight"] is None else z * one["post_weight"]
        z = z if one["gate"] is None else z * spread(one["gate"], c, len(z))
        sx = sx + abs(c["alpha"]) * z
    if c["norm"] == "none":
        return sx, None
    # an error of x_out passes through the norm: at most twice its share, over the deviation
    dev = x - x.mean(1, keepdim=True) if c["norm"] == "layer" else x
    r = 1 / (dev.pow(2).mean(1, keepdim=True) + c["eps"]).sqrt()
    rms = sx.pow(2).mean(1, keepdim=True).sqrt()
    sh = size_of_norm(x, c["norm"], c["eps"]) + (sx + rms + normed(x, c["norm"], c["eps"]).abs() * rms) * r
    sh = sh if one["weight"] is None else sh * one["weight"]
    sh = sh if one["bias"] is None else sh + one["bias"]
    sh = sh if one["scale"] is None else sh * (1 + spread(one["scale"], c, len(sh)))
    return sx, sh if one["shift"] is None else sh + spread(one["shift"], c, len(sh))


def to_gpu(t):
    return {k: None if v is None else v.to(DEV) for k, v in t.items()}


def check(got, want, tol, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - want).abs() / tol).max().item() if want.numel() else 0.0
    assert over <= 1.0, f"{what}: {over:.3f} of the tolerance"


FORWARD = [
    # one row, one chunk, the widest row, row widths at the borders of a wave's and a workgroup's share
    make(1, 8), make(1, 16384, x=BF16, norm="rms", weight=True), make(2, 504), make(3, 512, norm="rms"),
    make(5, 520, scale=True, shift=True, group=2), make(7, 1536, gate=True, scale=True, shift=True, group=3),
    make(4, 2048, post="rms", post_weight=True), make(3, 2056, post="layer", gate=True, group=1),
    make(2, 5120, x=BF16, post="rms", post_weight=True, gate=True, weight=True, bias=True, scale=True, shift=True),
    make(2, 8192, norm="rms", scale=True), make(3, 16376, shift=True, bias=True),
    # heads as rows (many rows of one chunk group), odd counts of rows
    make(1031, 64, x=BF16, norm="rms", weight=True, y=None), make(257, 128, y=None, h=F32), make(33, 24, y=F32, h=F32),
    # the stream alone
    make(9, 72, norm="none", gate=True, group=4), make(6, 640, norm="none", post="layer", post_weight=True, x=BF16),
    # groups: one row each, more rows than there are, a short last one
    make(10, 96, scale=True, gate=True, group=1), make(10, 96, shift=True, group=100), make(11, 96, scale=True, group=5),
    make(700, 1536, x=BF16, y=F32, h=F32, gate=True, scale=True, shift=True, group=300),
]


@pytest.mark.parametrize("case", range(len(FORWARD)))
def test_forward(case):
    c, t, h_dtype = FORWARD[case]
    print(f"norm_residual {tuple(t['x'].shape)} {c}", flush=True)
    x_out, h = ispa.norm_residual(**to_gpu(t), **c, h_dtype=h_dtype)
    torch.cuda.synchronize()
    w = wide(t)
    x = stream(c, w)
    sx, sh = sizes(c, w, x)
    check(x_out, x, x.abs() * half_step(t["x"].dtype) + sx * ROW + 1e-30, "x_out")
    assert x_out.dtype == t["x"].dtype
    if c["norm"] == "none":
        assert h is None
        return
    want = head(c, w, x)
    assert h.dtype == h_dtype
    check(h, want, want.abs() * half_step(h_dtype) + sh * ROW + 1e-30, "h")


BACKWARD = [
    make(1, 8), make(1, 16384, x=BF16, norm="rms", weight=True), make(3, 512, norm="rms", weight=True, bias=True),
    make(37, 520, scale=True, shift=True, group=2), make(70, 1536, gate=True, scale=True, shift=True, group=30),
    make(64, 2048, post="rms", post_weight=True, weight=True), make(40, 2056, post="layer", gate=True, group=1),
    make(50, 5120, x=BF16, post="rms", post_weight=True, gate=True, weight=True, bias=True, scale=True, shift=True,
         group=20),
    make(1031, 64, x=BF16, norm="rms", weight=True, y=None), make(257, 128, y=None, h=F32, bias=True),
    make(33, 24, y=F32, h=F32, post="layer", post_weight=True, gate=True),
    make(90, 72, norm="none", gate=True, group=4), make(60, 640, norm="none", post="layer", post_weight=True, x=BF16),
    make(10, 96, scale=True, gate=True, group=1), make(11, 96, scale=True, weight=True, bias=True, group=5),
    make(900, 96, scale=True, shift=True, weight=True, bias=True, gate=True, group=7),
    make(5, 1024), make(700, 1536, x=BF16, y=F32, h=F32, gate=True, scale=True, group=300),
    # every vector over one group: of few rows, of many, and with a group length behind them
    make(3, 40, post="rms", post_weight=True, gate=True, weight=True, bias=True, scale=True, shift=True),
    make(700, 1536, post="layer", post_weight=True, gate=True, weight=True, bias=True, scale=True, shift=True),
    make(2000, 64, x=BF16, y=F32, norm="rms", post="rms", post_weight=True, gate=True, weight=True, scale=True, group=4000),
    # twelve waves to a row, sixteen, and two chunks to a lane of ten, of thirteen and sixteen waves
    make(600, 6144, post="rms", post_weight=True, scale=True, group=150), make(520, 8192, gate=True, weight=True, bias=True),
    make(300, 10240, x=BF16, y=F32, scale=True, group=200), make(270, 13000, norm="rms", post="layer", weight=True),
    make(260, 16376, x=BF16, h=F32, gate=True, shift=True),
]


@pytest.mark.parametrize("direct", [True, False])
@pytest.mark.parametrize("case", range(len(BACKWARD)))
def test_backward(case, direct):
    c, t, h_dtype = BACKWARD[case]
    if c["norm"] == "none" and not direct:
        pytest.skip("without a norm nothing else reaches the stream")
    rows, cols = t["x"].shape
    g = torch.Generator().manual_seed(case)
    d_h = torch.randn(rows, cols, generator=g).to(h_dtype) if c["norm"] != "none" else None
    d_x = torch.randn(rows, cols, generator=g).to(t["x"].dtype) if direct else None
    print(f"norm_residual_backward {(rows, cols)} {c}", flush=True)
    gpu = to_gpu(t)
    x_gpu = gpu.pop("x")
    got = ispa.norm_residual_backward(None if d_h is None else d_h.to(DEV), x_gpu,
                                      d_x_out=None if d_x is None else d_x.to(DEV), **gpu, **c)
    torch.cuda.synchronize()
    # x is the stream after the block here: the branch is differentiated on its own
    w = wide(t, grad=True)
    wrt = [k for k in ("x", "weight", "bias", "scale", "shift") if w[k] is not None]
    want, gx = {}, torch.zeros(rows, cols, dtype=torch.float64)
    if d_h is not None:
        grads = torch.autograd.grad((head(c, w, w["x"]) * d_h.double()).sum(), [w[k] for k in wrt])
        want = dict(zip(wrt, grads))
        gx = want["x"]
    want["x"] = gx + (d_x.double() if direct else 0)
    if w["y"] is not None:
        wrt = [k for k in ("y", "post_weight", "gate") if w[k] is not None]
        branch = stream(c, {**w, "x": torch.zeros(rows, cols, dtype=torch.float64)})
        want.update(zip(wrt, torch.autograd.grad((branch * want["x"].detach()).sum(), [w[k] for k in wrt])))
    want = {k: v.detach() for k, v in want.items()}
    assert set(got) == set(want)
    w = wide(t)

    # the magnitudes that enter each gradient
    sd = torch.zeros(rows, cols, dtype=torch.float64) if d_x is None else d_x.double().abs()
    sums = lambda v: torch.stack([v[i:i + (c["group_rows"] or rows)].sum(0) for i in range(0, rows, c["group_rows"] or rows)])
    size = {}
    if d_h is not None:
        xh, sx = normed(w["x"], c["norm"], c["eps"]), size_of_norm(w["x"], c["norm"], c["eps"])
        dh = d_h.double().abs()
        du = dh if w["scale"] is None else dh * (1 + spread(w["scale"].abs(), c, rows))
        size.update(shift=sums(dh), scale=sums(dh * ((sx if w["weight"] is None else sx * w["weight"].abs())
                                                     + (0 if w["bias"] is None else w["bias"].abs()))),
                    weight=(du * sx).sum(0), bias=du.sum(0))
        gu = du if w["weight"] is None else du * w["weight"].abs()
        dev = w["x"] - w["x"].mean(1, keepdim=True) if c["norm"] == "layer" else w["x"]
        r = 1 / (dev.pow(2).mean(1, keepdim=True) + c["eps"]).sqrt()
        # (an error of r or of xhat enters twice)
        sd = sd + 4 * r * (gu + gu.mean(1, keepdim=True) + sx * (gu * sx).mean(1, keepdim=True))
    size["x"] = sd
    if w["y"] is not None:
        sy = size_of_norm(w["y"], c["post"], c["eps"])
        a = abs(c["alpha"])
        gate = 1 if w["gate"] is None else spread(w["gate"].abs(), c, rows)
        pw = 1 if w["post_weight"] is None else w["post_weight"].abs()
        size.update(gate=sums(a * sd * sy * pw), post_weight=(a * sd * gate * sy).sum(0))
        gz = a * sd * gate * pw
        if c["post"] == "none":
            size["y"] = gz
        else:
            dev = w["y"] - w["y"].mean(1, keepdim=True) if c["post"] == "layer" else w["y"]
            r = 1 / (dev.pow(2).mean(1, keepdim=True) + c["eps"]).sqrt()
            size["y"] = 4 * r * (gz + gz.mean(1, keepdim=True) + sy * (gz * sy).mean(1, keepdim=True))
    for k, v in want.items():
        dtype = t[k].dtype
        assert got[k].dtype == dtype
        tol = v.abs() * half_step(dtype) + size[k] * (ROW if k in ("x", "y") else COL) + 1e-30
        check(got[k], v, tol, k)


@pytest.mark.parametrize("cols", [64, 1024, 2056])
def test_backward_without_eps(cols):
    # eps 0 is allowed where no row is constant; slots without a row must not reach the sums
    c, t, _ = make(5, cols, norm="rms", post="layer", post_weight=True, weight=True, gate=True, scale=True, group=2)
    c["eps"] = 0.0
    gpu = to_gpu(t)
    d_h = torch.randn(5, cols, generator=torch.Generator().manual_seed(cols)).to(BF16)
    x_gpu = gpu.pop("x")
    got = ispa.norm_residual_backward(d_h.to(DEV), x_gpu, **gpu, **c)
    w = wide(t, grad=True)
    want = torch.autograd.grad((head(c, w, w["x"]) * d_h.double()).sum(), [w["weight"], w["scale"], w["x"]])
    branch = stream(c, {**w, "x": torch.zeros(5, cols, dtype=torch.float64)})
    gate, pw = torch.autograd.grad((branch * want[2]).sum(), [w["gate"], w["post_weight"]])
    # sums of at most five terms of order ten: 2^-18 of their magnitudes
    for name, v in (("weight", want[0]), ("scale", want[1]), ("gate", gate), ("post_weight", pw)):
        check(got[name], v.detach(), 2.0 ** -12 * (1 + v.detach().abs()), name)


def test_gradient_against_differences():
    # the backward pass against central differences of the forward pass in fp32: a step of
    # 2^-6 leaves a relative second-order error below 2^-8 and a rounding of 2^-18 / 2^-6
    c, t, _ = make(6, 64, y=F32, h=F32, gate=True, scale=True, shift=True, weight=True, bias=True, post="rms",
                   post_weight=True, group=4, seed=3)
    t["x"] = torch.randn(6, 64, generator=torch.Generator().manual_seed(1))
    gpu = to_gpu(t)
    g = torch.Generator().manual_seed(2)
    d_h, d_x = torch.randn(6, 64, generator=g).to(DEV), torch.randn(6, 64, generator=g).to(DEV)
    x_out, _ = ispa.norm_residual(**gpu, **c, h_dtype=F32)
    rest = {k: v for k, v in gpu.items() if k != "x"}
    grads = ispa.norm_residual_backward(d_h, x_out, d_x_out=d_x, **rest, **c)

    def loss(**kw):
        x, h = ispa.norm_residual(**{**gpu, **kw}, **c, h_dtype=F32)
        return (x.double() * d_x.double()).sum() + (h.double() * d_h.double()).sum()

    for name, v in gpu.items():
        way = torch.randn(v.shape, generator=g).to(DEV)
        way = way / way.norm()
        step = 2.0 ** -6
        slope = ((loss(**{name: v + step * way}) - loss(**{name: v - step * way})) / (2 * step)).item()
        want = (grads[name].double() * way.double()).sum().item()
        scale = grads[name].double().norm().item()
        assert abs(slope - want) <= 2.0 ** -8 * scale + 1e-3, (name, slope, want)


def test_in_place_and_given_outputs():
    c, t, _ = make(37, 256, gate=True, scale=True, shift=True, group=10)
    gpu = to_gpu(t)
    x_out, h = ispa.norm_residual(**gpu, **c)
    x2, h2 = gpu["x"].clone(), torch.empty_like(h)
    a, b = ispa.norm_residual(**{**gpu, "x": x2}, **c, x_out=x2, h=h2)
    assert a is x2 and b is h2
    assert torch.equal(x_out, x2) and torch.equal(h, h2)
    same, h3 = ispa.norm_residual(gpu["x"], norm="rms")
    assert same is gpu["x"]
    with pytest.raises(ispa.IspaError):
        ispa.norm_residual(gpu["x"], gpu["x"], x_out=gpu["x"])     # x_out over y
    with pytest.raises(ValueError):
        ispa.norm_residual(gpu["x"], gpu["y"][:5])
    with pytest.raises(ValueError):
        ispa.norm_residual(gpu["x"], scale=gpu["scale"])           # one group of rows, three vectors
    with pytest.raises(ValueError):
        ispa.norm_residual(gpu["x"].t())
    with pytest.raises(ispa.IspaError):
        ispa.norm_residual(torch.zeros(4, 12, device=DEV))         # columns not a multiple of 8


def test_empty_and_non_finite_rows():
    x, h = ispa.norm_residual(torch.zeros(0, 64, device=DEV), torch.zeros(0, 64, device=DEV))
    assert x.shape == (0, 64) and h.shape == (0, 64)
    g = ispa.norm_residual_backward(h, x, weight=torch.ones(64, device=DEV))
    assert g["x"].shape == (0, 64) and not g["weight"].any()
    # a row of zeros gives zeros, one of NaN or infinities nothing finite, the others are not touched by it
    x = torch.randn(9, 1536, device=DEV)
    want = ispa.norm_residual(x, h_dtype=F32)[1]
    bad = x.clone()
    bad[2], bad[4, 7], bad[6, 0] = 0.0, float("nan"), float("inf")
    h = ispa.norm_residual(bad, h_dtype=F32)[1]
    keep = [0, 1, 3, 5, 7, 8]
    assert torch.equal(h[keep], want[keep])
    assert not h[2].any() and torch.isnan(h[4]).all() and torch.isnan(h[6, 0])


def test_repeats_streams_and_graph():
    # the same bits again, on another stream, and in a graph replayed over new values
    c, t, _ = make(300, 1536, gate=True, scale=True, shift=True, weight=True, group=128)
    gpu = to_gpu(t)
    d_h = torch.randn(300, 1536, device=DEV).to(BF16)
    rest = {k: v for k, v in gpu.items() if k != "x"}

    def both():
        x, h = ispa.norm_residual(**gpu, **c)
        return [x, h] + [v for _, v in sorted(ispa.norm_residual_backward(d_h, x, **rest, **c).items())]

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = both()
    for turn in range(3):
        gpu["x"].copy_(torch.randn(300, 1536, device=DEV))
        gpu["gate"].mul_(1.5)
        want = both()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, kept)), turn


def test_a_short_last_group_of_very_many_rows():
    # 2^22 - 1 rows in a group of all but one and a group of one: the grid counts the rows, not
    # twice the long group's (whose 2^23 workgroups of nine waves no launch holds)
    rows, cols = (1 << 22) - 1, 8200
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GB of free device memory")
    x = torch.empty(rows, cols, dtype=BF16, device=DEV)
    row = torch.randn(3, cols, generator=torch.Generator().manual_seed(5)).to(BF16)
    at = [0, 1, rows // 2, rows - 2, rows - 1]
    x.copy_(row[2].to(DEV).expand(rows, cols))
    x[at[:4]] = row[[0, 1, 0, 1]].to(DEV)
    scale = torch.randn(2, cols, generator=torch.Generator().manual_seed(6))
    h = torch.empty_like(x)
    _, h = ispa.norm_residual(x, scale=scale.to(DEV), group_rows=rows - 1, h=h)
    torch.cuda.synchronize()
    got, want_x = h[at].double().cpu(), row[[0, 1, 0, 1, 2]].double()
    want = normed(want_x, "layer", 1e-6) * (1 + scale.double()[[0, 0, 0, 0, 1]])
    size = size_of_norm(want_x, "layer", 1e-6) * (1 + scale.double().abs()[[0, 0, 0, 0, 1]])
    check(got, want, want.abs() * half_step(BF16) + size * ROW, "h")
    del x, h
    torch.cuda.empty_cache()
