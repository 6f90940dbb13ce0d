"""Cosine and sine of norm_rotary to the last bit of fp32: heads whose rms is 1, with one value of
each turned pair 2 or 0 and the other 0, give 2 cos and 2 sin of the angles themselves. Angles, cosine,
sine and amplitude are fp64 and rounded once, 2^-24 of the value; the fp64 steps are off by less than
2^-48."""

import pytest
import torch

import paper_2607_00712_amd as ispa

pytestmark = pytest.mark.gpu
DEV = "cuda"


def heads(rows, d, rotary, interleaved):
    """Two heads [rows, 2, d]: the first pairs' first value 2 in d / 4 of them, the others 0."""
    x = torch.zeros(rows, 2, d)
    half = rotary // 2
    for h in range(2):
        j = torch.arange(h * (half - d // 4), h * (half - d // 4) + d // 4)
        x[:, h, 2 * j if interleaved else j] = 2.0
    assert (x.square().mean(-1) == 1).all()
    return x


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d, far, amplitude", [(128, 1, 1.0), (64, 4000, 1.25), (128, 1000003, 1.2772588), (256, 2 ** 31 - 6000, 1.0)])
def test_angles(d, far, amplitude, interleaved):
    rows, half = 70, d // 2
    x = heads(rows, d, d, interleaved)
    g = torch.Generator().manual_seed(d)
    p = torch.randint(0, 5000, (rows, 1), generator=g, dtype=torch.int32) + (far if far > 1 else 0)
    f = ispa.rotary_frequencies(half, device="cpu")[0]
    amplitude = float(torch.tensor(amplitude))  # (an fp32 argument)
    angle = p.double() * f
    c, s = angle.cos()[:, None] * amplitude, angle.sin()[:, None] * amplitude
    i, k = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, half), slice(half, None))

    def check(got, want, what):
        over = (got.cpu().double() - want).abs() - (want.abs() * 2.0 ** -24 + 2.0 ** -48)
        assert torch.all(over <= 0), f"{what}: {over.max().item():.3e} over the tolerance"

    put = lambda t: t.flatten(1).to(DEV)
    q, none = ispa.norm_rotary(put(x), None, p.to(DEV), f.to(DEV), 2, norm="rms", eps=0.0, interleaved=interleaved,
                               amplitude=amplitude)
    want = torch.zeros(x.shape, dtype=torch.float64)
    want[..., i], want[..., k] = x[..., i] * c, x[..., i] * s
    check(q.view(x.shape), want, "turned")
    # the gradient turns the other way; db is its sum over one row and head
    for r in (0, rows - 1):
        back = ispa.norm_rotary_backward(put(x[r:r + 1, :1]), None, put(x[r:r + 1, :1]), None, p[r:r + 1].to(DEV), f.to(DEV), 1,
                                         norm="rms", eps=0.0, q_bias=torch.zeros(d, device=DEV), interleaved=interleaved,
                                         amplitude=amplitude)
        want = torch.zeros(d, dtype=torch.float64)
        want[i], want[k] = x[r, 0, i] * c[r, 0], -x[r, 0, i] * s[r, 0]
        check(back["q_bias"], want, "gradient")
