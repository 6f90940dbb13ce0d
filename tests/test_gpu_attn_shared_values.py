"""attn_shared where a bound that fits every call says little.

Tolerances. The scores' error e, and B = sum w_i |v_i| + |O|, are those of
test_gpu_attn_shared.py (`exact` there gives (2^-8 + 2 e + 2^-20) B as the tolerance of
weights rounded to bf16). Weights of two bf16 parts are within 2^-16: the first part
leaves at most 2^-8 of a weight, the second rounds that by 2^-8. The products' sums in
fp32 may lose a step at each key, n 2^-23; an exponent and the reference that it is taken
against are each rounded at their own size, at most |s| log2 e 2^-24 each, and the
exponential itself within two steps: with |s| <= 12, less than 2^-17.
"""

import pytest
import torch

import paper_2607_00712_amd as ispa
from test_gpu_attn_shared import exact, make, on_gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def small(case, **kw):
    """Inputs whose scores are small, so that their own rounding (e) stays below the weights'."""
    counts, lens, prefix, capacity, heads, kv_heads, d = case
    return make(counts, lens, prefix, capacity, heads, kv_heads, d, q_scale=0.25, **kw)


def tight(t, heads, kv_heads):
    """exact() with the tolerance of weights of 16 bits."""
    out, _, tol, _ = exact(t, heads, kv_heads)
    d = t["q"].shape[1] // heads
    q = t["q"].double().nan_to_num().abs().view(-1, heads, d)
    keys = torch.cat((t["k_prefix"], t["k_cache"].flatten(0, 1))).double().abs().view(-1, kv_heads, d)
    most = max((q[:, h] @ keys[:, h // (heads // kv_heads)].t()).max().item() for h in range(heads)) / d ** 0.5
    assert most <= 12
    e = (d + 8) * 2.0 ** -24 * most
    b = tol / (2.0 ** -8 + 2.0 ** -20)          # B, or a little more
    n = len(t["k_prefix"]) + t["k_cache"].shape[1]
    return out, (2.0 ** -16 + 2 * e + n * 2.0 ** -23 + 2.0 ** -17) * b


def over(got, want, tol):
    """The largest error as a part of the tolerance."""
    return ((got.double().cpu() - want).abs() / (tol + 1e-30)).max().item()


# counts, own lengths, prefix, capacity, heads, kv_heads, head_dim: tiles of 32, 64, 128 rows
NARROW = [([3, 1], [40, 7], 120, 64, 2, 2, 64), ([5, 2], [33, 64], 130, 64, 8, 2, 128), ([40], [20], 140, 32, 1, 1, 128),
          ([30, 25], [64, 5], 120, 64, 2, 2, 64), ([50, 50], [30, 31], 130, 64, 2, 2, 128),
          ([30, 60], [40, 1], 120, 40, 3, 3, 64)]
# and wider ones, of the batch or of a request
WIDE = [([200, 70], [40, 7], 120, 64, 2, 2, 64), ([300], [33], 130, 64, 4, 2, 128), ([60, 1, 40], [33, 0, 64], 130, 64, 6, 2, 128),
        ([150, 3], [64, 64], 0, 64, 2, 1, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(NARROW) + len(WIDE)))
def test_weights_keep_16_bits(case):
    counts, lens, prefix, capacity, heads, kv_heads, d = (NARROW + WIDE)[case]
    t = small((NARROW + WIDE)[case])
    print(f"attn_shared fp32 {(NARROW + WIDE)[case]}", flush=True)
    out, _ = ispa.attn_shared(**on_gpu(t), n_heads=heads, n_kv_heads=kv_heads, out_dtype=F32, max_q=max(counts))
    torch.cuda.synchronize()
    share = over(out, *tight(t, heads, kv_heads))
    assert share <= 1, f"{share:.2f} of the tolerance"


@pytest.mark.gpu
@pytest.mark.parametrize("pad", [0, 500])
def test_padding_costs_no_accuracy(pad):
    # a few real rows in tensors of a fixed count of rows
    counts, _, _, _, heads, kv_heads, _ = NARROW[1]
    t = small(NARROW[1], pad=pad)
    real = sum(counts)
    out, _ = ispa.attn_shared(**on_gpu(t), n_heads=heads, n_kv_heads=kv_heads, out_dtype=F32)
    torch.cuda.synchronize()
    want, tol = tight(t, heads, kv_heads)
    share = over(out[:real], want[:real], tol[:real])
    assert share <= 1, f"{share:.2f} of the tolerance"


@pytest.mark.parametrize("case", range(len(NARROW) + len(WIDE)))
def test_the_bound_tells_8_bits_from_16(case):
    # the definition with its weights rounded to bf16 does not pass
    counts, lens, prefix, capacity, heads, kv_heads, d = (NARROW + WIDE)[case]
    t = small((NARROW + WIDE)[case])
    want, tol = tight(t, heads, kv_heads)
    got, starts = want.clone(), t["q_start"].tolist()
    for b, n in enumerate(lens):
        at = slice(starts[b], starts[b + 1])
        k, v = (torch.cat((t[f"{x}_prefix"], t[f"{x}_cache"][b, :n])).double() for x in "kv")
        for h in range(heads):
            c = h // (heads // kv_heads) * d
            s = t["q"][at, h * d:(h + 1) * d].double() @ k[:, c:c + d].t() / d ** 0.5
            w = (s - s.amax(1, keepdim=True)).exp().to(BF16).double()
            got[at, h * d:(h + 1) * d] = (w / w.sum(1, keepdim=True)) @ v[:, c:c + d]
    assert over(got, want, tol) > 1.5
