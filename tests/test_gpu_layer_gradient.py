"""A training step through the norms and the positions around a layer's attention, as a
program writes it: the calls and their gradients as autograd functions, with torch's
products between them, against autograd of the same in 64 bits.

Everything is fp32. A norm's outputs and gradients are within 2^-18 of the magnitudes that
enter them, a turned value within 2^-21, a product over 192 values within 192 x 2^-24 <
2^-16; the vectors' gradients sum 37 rows on top of that. Each stage is linear in what the
one before is off by, with factors of order one for these inputs (deviations near one,
weights of the size 1 / sqrt(192)); magnitudes exceed results by at most sqrt(192) < 2^4
where terms cancel: three products and four calls in turn stay below 7 x 2^4 x 2^-16 <
2^-9 of a gradient's 2-norm.
"""

import pytest
import torch

import paper_2607_00712_amd as ispa

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32 = torch.float32


class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, weight, scale, shift, gate, post_weight, how):
        v = dict(weight=weight, scale=scale, shift=shift, gate=gate, post_weight=post_weight)
        x_out, h = ispa.norm_residual(x, y, **v, **how, h_dtype=F32)
        ctx.save_for_backward(x_out, y, *v.values())
        ctx.how = how
        return x_out, h

    @staticmethod
    def backward(ctx, d_x_out, d_h):
        x_out, y, *v = ctx.saved_tensors
        names = ("weight", "scale", "shift", "gate", "post_weight")
        g = ispa.norm_residual_backward(d_h.contiguous(), x_out, y, d_x_out=d_x_out.contiguous(), **dict(zip(names, v)),
                                        **ctx.how)
        return g["x"], g["y"], *(g[n] for n in names), None


class Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, freqs, heads, how):
        ctx.save_for_backward(positions, freqs)
        ctx.heads, ctx.how = heads, how
        return ispa.rotary(x, positions, freqs, heads, **how)

    @staticmethod
    def backward(ctx, d):
        return ispa.rotary(d.contiguous(), *ctx.saved_tensors, ctx.heads, inverse=True, **ctx.how), None, None, None, None


@pytest.mark.parametrize("norm, post, interleaved", [("layer", "rms", True), ("rms", "layer", False)])
def test_gradients_through_a_layer(norm, post, interleaved):
    rows, cols, heads, d, group = 37, 192, 3, 64, 10
    groups = -(-rows // group)
    g = torch.Generator().manual_seed(len(norm))
    r = lambda *s: torch.randn(*s, generator=g)
    leaves = dict(x=r(rows, cols), y=r(rows, cols), weight=1 + 0.2 * r(cols), scale=0.2 * r(groups, cols),
                  shift=0.2 * r(groups, cols), gate=r(groups, cols), post_weight=1 + 0.2 * r(cols),
                  w_q=r(cols, cols) / cols ** 0.5, w_o=r(cols, cols) / cols ** 0.5)
    how = dict(norm=norm, post=post, alpha=0.5, group_rows=group, eps=1e-6)
    p = torch.randint(0, 4000, (rows, 2), generator=g, dtype=torch.int32)
    axes, amplitude = (16, 8), 1.1                      # 48 of a head's 64 values turn
    f, _ = ispa.rotary_frequencies(axes, device="cpu")
    c, e = r(rows, cols), r(rows, cols)

    # the calls
    t = {k: v.to(DEV).requires_grad_(True) for k, v in leaves.items()}
    turn = lambda q: Rotary.apply(q, p.to(DEV), f.to(DEV), heads, dict(axes=axes, interleaved=interleaved,
                                                                       amplitude=amplitude))
    vectors = [t[k] for k in ("weight", "scale", "shift", "gate", "post_weight")]
    x_out, h = Norm.apply(t["x"], t["y"], *vectors, how)
    z = turn(h @ t["w_q"]) @ t["w_o"]
    x2, h2 = Norm.apply(x_out, z, *vectors, how)        # the same vectors again: their gradients add up
    ((h2 * c.to(DEV)).sum() + (x2 * e.to(DEV)).sum()).backward()
    torch.cuda.synchronize()

    # the same in 64 bits
    w = {k: v.double().requires_grad_(True) for k, v in leaves.items()}

    def normed(v, kind):
        v = v - v.mean(1, keepdim=True) if kind == "layer" else v
        return v / (v.pow(2).mean(1, keepdim=True) + 1e-6).sqrt()

    spread = lambda v: v.repeat_interleave(group, dim=0)[:rows]

    def block(x, y):
        x = x + 0.5 * spread(w["gate"]) * normed(y, post) * w["post_weight"]
        return x, normed(x, norm) * w["weight"] * (1 + spread(w["scale"])) + spread(w["shift"])

    axis = torch.tensor([k for k, n in enumerate(axes) for _ in range(n)])
    angle = (p.double()[:, axis] * f)[:, None]

    def turned(q):
        q, half = q.view(rows, heads, d), len(f)
        a, b, rest = ((q[..., 0:2 * half:2], q[..., 1:2 * half:2], q[..., 2 * half:]) if interleaved else
                      (q[..., :half], q[..., half:2 * half], q[..., 2 * half:]))
        a, b = amplitude * (a * angle.cos() - b * angle.sin()), amplitude * (a * angle.sin() + b * angle.cos())
        ab = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
        return torch.cat((ab, rest), -1).flatten(1)

    X, H = block(w["x"], w["y"])
    X2, H2 = block(X, turned(H @ w["w_q"]) @ w["w_o"])
    ((H2 * c.double()).sum() + (X2 * e.double()).sum()).backward()
    for k in leaves:
        want = w[k].grad
        off = ((t[k].grad.double().cpu() - want).norm() / want.norm()).item()
        assert off <= 2.0 ** -9, (k, off)
