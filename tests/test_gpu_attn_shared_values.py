"""attn_shared where a bound that fits every call says little: the weights' 16 bits, every
block of values, batches of more row tiles than the plan lists, tiles that take turns.

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


def stripe(t, kv_heads):
    """Block i of 32 values is seen in every s-th channel from i % s on alone, s the blocks or the
    channels of a head: a channel is the sum of few blocks, and a wrong one shows."""
    for name in ("v_prefix", "v_cache"):
        v = t[name]
        keys = v.shape[-2]
        d = v.shape[-1] // kv_heads
        blocks = -(-keys // 32)
        if blocks == 0:
            continue
        s = min(blocks, d)
        seen = (torch.arange(keys)[:, None] // 32 % s) == (torch.arange(d)[None] % s)
        t[name] = (v.view(*v.shape[:-1], kv_heads, d) * seen[:, None]).flatten(-2)
    return t


# counts, own lengths, prefix, capacity, heads, kv_heads, head_dim
STRIPED = [
    ([1] * 5, [3000, 0, 1, 2999, 512], 20011, 3000, 2, 2, 128), ([2], [7000], 9001, 7001, 1, 1, 64),
    ([3, 30], [700, 1000], 2500, 1001, 2, 1, 128), ([50, 50], [90, 64], 1700, 100, 2, 2, 64),
    ([130, 70, 200], [300, 0, 17], 1901, 300, 2, 2, 128), ([300, 9], [33, 1200], 2501, 1200, 2, 1, 64),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(STRIPED)))
def test_every_block_of_values(case):
    counts, lens, prefix, capacity, heads, kv_heads, d = STRIPED[case]
    t = stripe(make(counts, lens, prefix, capacity, heads, kv_heads, d), kv_heads)
    print(f"attn_shared striped {STRIPED[case]}", flush=True)
    out, _ = ispa.attn_shared(**on_gpu(t), n_heads=heads, n_kv_heads=kv_heads, max_q=max(counts))
    torch.cuda.synchronize()
    want, _, tol, _ = exact(t, heads, kv_heads)
    share = over(out, want, tol + 2.0 ** -8 * want.abs())
    assert share <= 1, f"{share:.2f} of the tolerance"


@pytest.mark.parametrize("case", [0, 1, 5])
@pytest.mark.parametrize("wrong", ["zero", "reversed", "next", "channels"])
def test_a_wrong_block_of_values_shows(case, wrong):
    counts, lens, prefix, capacity, heads, kv_heads, d = STRIPED[case]
    counts = [min(m, 4) for m in counts]
    t = stripe(make(counts, lens, prefix, capacity, heads, kv_heads, d), kv_heads)
    want, _, tol, _ = exact(t, heads, kv_heads)
    blocks = -(-prefix // 32)
    for i in (0, 1, blocks // 7, blocks // 2, blocks - 2):
        v = t["v_prefix"].clone()
        at = slice(32 * i, 32 * i + 32)
        if wrong == "zero":
            v[at] = 0
        elif wrong == "reversed":
            v[at] = v[at].flip(0)
        elif wrong == "next":
            v[at][:len(v[32 * i + 32:32 * i + 64])] = v[32 * i + 32:32 * i + 64]
        else:
            v[at] = v[at].roll(8, 1)
        got, _, _, _ = exact({**t, "v_prefix": v}, heads, kv_heads)
        assert over(got, want, tol + 2.0 ** -8 * want.abs()) > 1, (wrong, i)


@pytest.mark.gpu
@pytest.mark.parametrize("real", [1008, 1024, 1025, 1100, 9])
def test_more_row_tiles_than_plans(real):
    # 16 query heads to a key head: 69 tiles of 256 rows in the tensors, 63, 64, 65, 69 and 1 of real rows
    heads, kv_heads, d = 16, 1, 64
    counts = [real - 5, 5]
    t = stripe(make(counts, [17, 40], 3000, 40, heads, kv_heads, d, pad=1100 - real), kv_heads)
    out = torch.full((1100, heads * d), 4.0, dtype=BF16, device=DEV)
    lse = torch.full((heads, 1100), 6.0, device=DEV)
    print(f"attn_shared {real} of 1100 rows", flush=True)
    ispa.attn_shared(**on_gpu(t), n_heads=heads, n_kv_heads=kv_heads, max_q=max(counts), out=out, lse=lse)
    torch.cuda.synchronize()
    want, want_lse, tol, lse_tol = exact(t, heads, kv_heads)
    assert over(out[:real], want[:real], tol[:real] + 2.0 ** -8 * want[:real].abs()) <= 1
    assert over(lse[:, :real], want_lse[:, :real], lse_tol[:, :real]) <= 1
    assert (out[real:] == 4).all() and (lse[:, real:] == 6).all()


@pytest.mark.gpu
def test_row_tiles_take_turns():
    # 2048 requests of 8 key heads leave room for 128 row tiles of a request in the grid:
    # one request of 129 (33000 rows), the others of a row or none
    heads, d, n_req = 8, 64, 2048
    counts = [1 if b % 3 == 0 else 0 for b in range(n_req)]
    counts[7] = 33000
    lens = [b % 9 for b in range(n_req)]
    lens[7] = 8
    t = make(counts, lens, 33, 8, heads, heads, d)
    out, lse = ispa.attn_shared(**on_gpu(t), n_heads=heads, max_q=33000)
    torch.cuda.synchronize()
    want, want_lse, tol, lse_tol = exact(t, heads, heads)
    assert over(out, want, tol + 2.0 ** -8 * want.abs()) <= 1
    assert over(lse, want_lse, lse_tol) <= 1


@pytest.mark.gpu
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_a_captured_batch_of_changing_rows(out_dtype):
    # tensors of a fixed count of rows, captured once: the real rows are read on the device, from
    # none to all, across every count of row tiles
    heads, kv_heads, d, rows = 4, 2, 64, 400
    t = make([rows - 50, 50], [60, 33], 900, 64, heads, kv_heads, d)
    gpu = on_gpu(t)
    out, lse = torch.empty(rows, heads * d, dtype=out_dtype, device=DEV), torch.empty(heads, rows, device=DEV)
    call = lambda: ispa.attn_shared(**gpu, n_heads=heads, n_kv_heads=kv_heads, max_q=rows, out=out, lse=lse)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for counts in ([350, 50], [0, 0], [3, 1], [0, 64], [100, 30], [1, 256], [200, 200]):
        starts = [0, counts[0], sum(counts)]
        real = starts[2]
        gpu["q_start"].copy_(torch.tensor(starts, dtype=torch.int32))
        out.fill_(4.0), lse.fill_(6.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        assert (got[real:] == 4).all() and (got_lse[:, real:] == 6).all()
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, got) and torch.equal(lse, got_lse), counts
        want, want_lse, tol, lse_tol = exact({**t, "q_start": torch.tensor(starts)}, heads, kv_heads)
        if real:
            assert over(got[:real], want[:real], tol[:real] + 2.0 ** -8 * want[:real].abs()) <= 1, counts
            assert over(got_lse[:, :real], want_lse[:, :real], lse_tol[:, :real]) <= 1, counts


@pytest.mark.gpu
def test_requests_that_share_one_cache():
    # a distance of 0 between requests: each reads its own length of the same rows
    t = make([2, 3, 1], [40, 9, 33], 70, 40, 2, 2, 64)
    t["k_cache"], t["v_cache"] = (t[x][:1].expand(3, 40, 128) for x in ("k_cache", "v_cache"))
    gpu = on_gpu({k: v for k, v in t.items() if "cache" not in k or "lens" in k})
    for x in ("k_cache", "v_cache"):
        gpu[x] = t[x][0].to(DEV)[None].expand(3, 40, 128)
        assert gpu[x].stride(0) == 0
    out, _ = ispa.attn_shared(**gpu, n_heads=2)
    torch.cuda.synchronize()
    want, _, tol, _ = exact(t, 2, 2)
    assert over(out, want, tol + 2.0 ** -8 * want.abs()) <= 1
