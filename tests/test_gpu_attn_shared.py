"""attn_shared on the GPU against softmax attention over each request's key set in 64 bits.

Tolerances. With w the exact weights, O = sum w_i v_i. The weights enter the product
rounded to bf16 (2^-8 relative) and are normalised by the rounded sum, so O is off by at
most 2^-8 sum w_i |v_i - O| <= 2^-8 (sum w_i |v_i| + |O|) =: 2^-8 B. A score is an fp32
sum of head_dim products: off by at most (head_dim + 8) 2^-24 max_i sum |q k_i| scale =:
e, which moves a weight by 2 e relative. The output rounds once more: |O| eps / 2. The
LSE is off by e, and 2^-20 (1 + |LSE|) covers the exponentials, the fp32 sums and the
joins (each below 2^-22).
"""

import math

import pytest
import torch

import paper_2607_00712_amd as ispa

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def make(counts, lens, prefix, capacity, heads, kv_heads, head_dim, pad=0, seed=0, q_scale=1.0):
    g = torch.Generator().manual_seed(seed + 13 * prefix + capacity + len(counts))
    r = lambda *s: torch.randn(*s, generator=g).to(BF16)
    kv = kv_heads * head_dim
    rows = sum(counts) + pad
    starts = [0]
    for m in counts:
        starts.append(starts[-1] + m)
    return dict(q=(torch.randn(rows, heads * head_dim, generator=g) * q_scale).to(BF16), k_prefix=r(prefix, kv),
                v_prefix=r(prefix, kv), k_cache=r(len(counts), capacity, kv), v_cache=r(len(counts), capacity, kv),
                q_start=torch.tensor(starts, dtype=torch.int32), cache_lens=torch.tensor(lens, dtype=torch.int32))


def on_gpu(t):
    return {k: v.to(DEV) for k, v in t.items()}


def exact(t, heads, kv_heads, scale=None):
    """out, lse and the tolerances of both (without the output's rounding)."""
    starts = t["q_start"].tolist()
    rows, hidden = t["q"].shape
    d = hidden // heads
    scale = 1 / math.sqrt(d) if scale is None else scale
    capacity = t["k_cache"].shape[1]
    out, tol = torch.zeros(rows, hidden, dtype=torch.float64), torch.zeros(rows, hidden, dtype=torch.float64)
    lse = torch.full((heads, rows), -math.inf, dtype=torch.float64)
    lse_tol = torch.zeros(heads, rows, dtype=torch.float64)
    for b, length in enumerate(t["cache_lens"].tolist()):
        at = slice(starts[b], starts[b + 1])
        n = min(max(length, 0), capacity)
        k = torch.cat((t["k_prefix"], t["k_cache"][b, :n])).double()
        v = torch.cat((t["v_prefix"], t["v_cache"][b, :n])).double()
        if not len(k) or at.start == at.stop:
            continue
        for h in range(heads):
            c = h // (heads // kv_heads)
            q = t["q"][at, h * d:(h + 1) * d].double()
            kh, vh = k[:, c * d:(c + 1) * d], v[:, c * d:(c + 1) * d]
            s = q @ kh.t() * scale
            w = torch.softmax(s, 1)
            o = w @ vh
            e = (d + 8) * 2.0 ** -24 * (q.abs() @ kh.abs().t()).amax(1) * abs(scale)
            out[at, h * d:(h + 1) * d] = o
            tol[at, h * d:(h + 1) * d] = (2.0 ** -8 + 2 * e[:, None] + 2.0 ** -20) * (w @ vh.abs() + o.abs())
            lse[h, at] = torch.logsumexp(s, 1)
            lse_tol[h, at] = e + 2.0 ** -20 * (1 + lse[h, at].abs())
    return out, lse, tol, lse_tol


def check(got, got_lse, want, what=""):
    out, lse, tol, lse_tol = want
    half = torch.finfo(got.dtype).eps / 2
    got, got_lse = got.double().cpu(), got_lse.double().cpu()
    rows = torch.isfinite(lse)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    assert torch.equal(torch.isfinite(got_lse), rows), f"{what}: lse"
    assert (got_lse[~rows] == -math.inf).all(), f"{what}: lse of empty rows"
    assert torch.all((got_lse - lse)[rows].abs() <= lse_tol[rows]), (
        f"{what}: lse {(got_lse - lse)[rows].abs().max():.3e}")
    over = (got - out).abs() - (tol + half * out.abs())
    assert torch.all(over <= 0), f"{what}: {over.max():.3e} over the tolerance"


# counts of rows, own lengths, prefix, capacity, heads, kv_heads, head_dim
CASES = [
    ([1], [0], 1, 1, 1, 1, 64), ([1], [1], 0, 1, 1, 1, 128), ([1, 1], [64, 0], 256, 64, 2, 2, 64),
    ([3, 0, 17, 1], [77, 5, 0, 33], 100, 77, 6, 2, 128), ([3, 0, 17, 1], [77, 5, 0, 33], 100, 77, 6, 2, 64),
    # keys that end around the blocks of 32 and the steps of 64 and 128
    ([1, 2, 1, 3], [31, 32, 33, 1], 31, 40, 4, 4, 128), ([1, 2, 1, 3], [63, 64, 65, 0], 33, 70, 4, 4, 64),
    ([1, 2, 1, 3], [127, 128, 129, 96], 65, 130, 4, 1, 128), ([2, 2], [5, 200], 129, 257, 8, 8, 128),
    # several segments of the prefix and of the own keys
    ([1] * 5, [3000, 0, 1, 2999, 512], 20011, 3000, 2, 2, 128), ([2], [7000], 9001, 7001, 1, 1, 64),
    # row tiles of 32, 64, 128 and 256 rows, and past them
    ([32], [40], 90, 64, 1, 1, 128), ([33], [40], 90, 64, 1, 1, 128), ([20, 20], [40, 64], 90, 64, 2, 2, 128),
    ([65], [40], 300, 64, 1, 1, 64), ([50, 50], [40, 64], 700, 64, 3, 1, 128), ([129], [40], 300, 64, 1, 1, 128),
    ([130, 70, 200], [300, 0, 17], 701, 300, 2, 2, 128), ([130, 70, 200], [300, 0, 17], 701, 300, 2, 1, 64),
    ([40, 1, 300], [33, 65, 129], 0, 129, 4, 2, 128), ([257, 3], [0, 0], 333, 50, 2, 2, 64),
    # the largest shares of query heads to a key head
    ([1, 1, 1], [9, 8, 7], 70, 9, 64, 1, 64), ([5, 4], [9, 8], 70, 9, 48, 3, 128),
    # requests without rows around ones with rows
    ([0, 0, 2, 0], [5, 5, 5, 5], 40, 6, 2, 2, 128),
]


@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_exact(case, out_dtype):
    counts, lens, prefix, capacity, heads, kv_heads, head_dim = CASES[case]
    t = make(counts, lens, prefix, capacity, heads, kv_heads, head_dim)
    print(f"attn_shared {CASES[case]}", flush=True)
    out, lse = ispa.attn_shared(**on_gpu(t), n_heads=heads, n_kv_heads=kv_heads, out_dtype=out_dtype, max_q=max(counts))
    torch.cuda.synchronize()
    assert out.dtype == out_dtype
    check(out, lse, exact(t, heads, kv_heads))


def test_no_keys_at_all():
    t = make([2, 1], [0, 3], 0, 4, 4, 2, 64)
    out, lse = ispa.attn_shared(**on_gpu(t), n_heads=4, n_kv_heads=2)
    torch.cuda.synchronize()
    assert not out[:2].any() and (lse[:, :2] == -math.inf).all()
    check(out, lse, exact(t, 4, 2))
    t = make([2, 1], [0, 0], 0, 0, 4, 2, 64)
    out, lse = ispa.attn_shared(**on_gpu(t), n_heads=4, n_kv_heads=2)
    assert not out.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("counts, pad", [([3, 2], 5), ([150, 40], 70), ([0, 0], 4)])
def test_padding_is_left_alone(counts, pad):
    t = make(counts, [20, 33], 75, 40, 4, 2, 128, pad=pad)
    gpu = on_gpu(t)
    real = sum(counts)
    gpu["q"][real:] = float("nan")
    out = torch.full((real + pad, 512), 4.0, dtype=BF16, device=DEV)
    lse = torch.full((4, real + pad), 6.0, device=DEV)
    ispa.attn_shared(**gpu, n_heads=4, n_kv_heads=2, out=out, lse=lse)
    torch.cuda.synchronize()
    assert (out[real:] == 4).all() and (lse[:, real:] == 6).all()
    want = exact(t, 4, 2)
    check(out[:real], lse[:, :real], tuple(w[:real] if i % 2 == 0 else w[:, :real] for i, w in enumerate(want)))


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("counts", [[1, 2], [60, 30], [200, 100]])
def test_whatever_lies_behind_the_keys(counts, head_dim):
    # NaN and infinities behind the filled rows and behind prefix_len; lengths beyond the
    # capacity (a ring's count of tokens) mean a full cache, negative ones an empty one
    t = make(counts, [37, 50], 101, 50, 2, 2, head_dim)
    gpu = on_gpu(t)
    for name in ("k", "v"):
        gpu[f"{name}_cache"][0, 37:] = float("nan") if name == "k" else float("inf")
        gpu[f"{name}_prefix"] = torch.cat((gpu[f"{name}_prefix"], torch.full((9, 2 * head_dim), float("nan"), dtype=BF16,
                                                                            device=DEV)))
    gpu["cache_lens"][1] = 1000
    out, lse = ispa.attn_shared(**gpu, n_heads=2, prefix_len=101)
    torch.cuda.synchronize()
    check(out, lse, exact(t, 2, 2))
    gpu["cache_lens"][0] = -3
    t["cache_lens"][0] = 0
    out, lse = ispa.attn_shared(**gpu, n_heads=2, prefix_len=101)
    check(out, lse, exact(t, 2, 2))


def test_a_bad_row_stays_alone():
    t = make([2, 2], [20, 30], 100, 30, 2, 2, 64)
    gpu = on_gpu(t)
    want, want_lse = ispa.attn_shared(**gpu, n_heads=2)
    gpu["q"][1, 3] = float("nan")
    gpu["k_cache"][1, 4, 64:] = float("inf")               # request 1's second head
    out, lse = ispa.attn_shared(**gpu, n_heads=2)
    torch.cuda.synchronize()
    assert torch.isnan(out[1, :64].float()).all() and torch.isnan(lse[0, 1])
    for rows, cols, head in ((slice(0, 1), slice(0, 128), slice(0, 2)), (slice(1, 2), slice(64, 128), slice(1, 2)),
                             (slice(2, 4), slice(0, 64), slice(0, 1))):
        assert torch.equal(out[rows, cols], want[rows, cols]) and torch.equal(lse[head, rows], want_lse[head, rows])


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("q_scale", [30.0, 1e-3])
def test_peaked_and_flat_weights(q_scale, head_dim):
    # one key far above the others (the reference moves late in the keys), and all equal
    t = make([4, 70], [100, 90], 400, 100, 2, 1, head_dim, q_scale=q_scale)
    out, lse = ispa.attn_shared(**on_gpu(t), n_heads=2, n_kv_heads=1)
    torch.cuda.synchronize()
    check(out, lse, exact(t, 2, 1))


def test_scores_far_below_zero_and_rising():
    # every score far below zero, and scores that rise with the key so that the softmax
    # reference moves in every block
    t = make([3], [64], 500, 64, 1, 1, 64)
    t["q"].fill_(4.0)
    ramp = torch.linspace(-50, -1, 500)[:, None].expand(500, 64)
    t["k_prefix"] = ramp.to(BF16).contiguous()
    t["k_cache"] = torch.full((1, 64, 64), -40.0).to(BF16)
    out, lse = ispa.attn_shared(**on_gpu(t), n_heads=1)
    torch.cuda.synchronize()
    check(out, lse, exact(t, 1, 1))


def test_scale_argument():
    t = make([3, 1], [5, 9], 77, 9, 2, 2, 64)
    out, lse = ispa.attn_shared(**on_gpu(t), n_heads=2, scale=0.5)
    torch.cuda.synchronize()
    check(out, lse, exact(t, 2, 2, 0.5))


@pytest.mark.parametrize("max_q", [None, 1, 7, 4096])
@pytest.mark.parametrize("counts", [[1, 1, 1], [50, 0, 1], [300, 2, 90]])
def test_max_q_is_a_hint(counts, max_q):
    t = make(counts, [60, 61, 3], 128, 61, 4, 2, 128)
    out, lse = ispa.attn_shared(**on_gpu(t), n_heads=4, n_kv_heads=2, max_q=max_q)
    torch.cuda.synchronize()
    check(out, lse, exact(t, 4, 2))


def test_strides():
    # q a slice of a wider product, keys and values interleaved in one cache, output a slice
    t = make([3, 9], [20, 33], 75, 40, 4, 2, 64)
    gpu = on_gpu(t)
    want, want_lse = ispa.attn_shared(**gpu, n_heads=4, n_kv_heads=2)
    both = torch.cat((gpu["k_cache"], gpu["v_cache"]), 2)
    prefix = torch.cat((gpu["v_prefix"], gpu["k_prefix"]), 1)
    wide = torch.cat((gpu["q"], gpu["q"] * 0, gpu["q"] * 2), 1)
    out = torch.full((12, 300 * 2), 2.0, dtype=BF16, device=DEV)
    _, lse = ispa.attn_shared(wide[:, :256], prefix[:, 128:], prefix[:, :128], both[..., :128], both[..., 128:],
                              gpu["q_start"], gpu["cache_lens"], 4, n_kv_heads=2, out=out[:, 8:264])
    torch.cuda.synchronize()
    assert torch.equal(out[:, 8:264], want) and torch.equal(lse, want_lse)
    assert (out[:, :8] == 2).all() and (out[:, 264:] == 2).all()
    for bad in (lambda: ispa.attn_shared(**{**gpu, "q": gpu["q"][:, :252]}, n_heads=4, n_kv_heads=2),
                lambda: ispa.attn_shared(**{**gpu, "k_cache": gpu["k_cache"][:, :5]}, n_heads=4, n_kv_heads=2),
                lambda: ispa.attn_shared(**gpu, n_heads=4, n_kv_heads=2, prefix_len=76),
                lambda: ispa.attn_shared(**{**gpu, "q_start": gpu["q_start"][:2]}, n_heads=4, n_kv_heads=2),
                lambda: ispa.attn_shared(**gpu, n_heads=4, n_kv_heads=3)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ispa.IspaError):
        ispa.attn_shared(**gpu, n_heads=4, n_kv_heads=2, out=gpu["q"])
    with pytest.raises(ispa.IspaError):
        ispa.attn_shared(**make_wrong_head_dim(), n_heads=2)


def test_output_beside_the_queries():
    # the output takes other columns of the rows that hold q; over q's own columns it is refused
    t = make([3, 9], [20, 33], 75, 40, 4, 2, 64)
    gpu = on_gpu(t)
    want, want_lse = ispa.attn_shared(**gpu, n_heads=4, n_kv_heads=2)
    wide = torch.cat((gpu["q"], gpu["q"] * 0), 1)
    args = {**gpu, "q": wide[:, :256]}
    _, lse = ispa.attn_shared(**args, n_heads=4, n_kv_heads=2, out=wide[:, 256:])
    torch.cuda.synchronize()
    assert torch.equal(wide[:, 256:], want) and torch.equal(lse, want_lse) and torch.equal(wide[:, :256], gpu["q"])
    with pytest.raises(ispa.IspaError):
        ispa.attn_shared(**args, n_heads=4, n_kv_heads=2, out=wide[:, 248:504])


def make_wrong_head_dim():
    return on_gpu(make([1], [2], 5, 3, 2, 2, 96))


@pytest.mark.parametrize("counts", [[2], [200]])
def test_offsets_behind_32_bits(counts):
    # prefix rows 2^23 elements apart (300 rows: 5 GB), own keys behind them
    t = make(counts, [7], 300, 8, 1, 1, 128)
    gpu = on_gpu(t)
    far = [torch.empty(300 * (1 << 23), dtype=BF16, device=DEV).view(300, 1 << 23) for _ in range(2)]
    for x, name in zip(far, ("k_prefix", "v_prefix")):
        x[:, :128] = gpu[name]
        gpu[name] = x[:, :128]
    out, lse = ispa.attn_shared(**gpu, n_heads=1)
    torch.cuda.synchronize()
    check(out, lse, exact(t, 1, 1))


def test_against_the_attention_of_one_request():
    # a batch of one request is the chunk attention over prefix and own keys in one cache
    t = make([70], [90], 500, 90, 4, 4, 128)
    gpu = on_gpu(t)
    out, lse = ispa.attn_shared(**gpu, n_heads=4, out_dtype=F32)
    k, v = (torch.cat((gpu[f"{n}_prefix"], gpu[f"{n}_cache"][0])) for n in ("k", "v"))
    ref, ref_lse = ispa.attn_chunk(gpu["q"], k, v, 590, 590, 4)
    _, lse64, tol, lse_tol = exact(t, 4, 4)
    assert torch.all((out - ref).abs().cpu() <= 2 * tol) and torch.all((lse - ref_lse).abs().cpu() <= 2 * lse_tol)


@pytest.mark.parametrize("counts", [[1] * 6, [90, 30, 0, 1, 2, 40]])
def test_repeats_streams_and_graph(counts):
    t = make(counts, [5, 100, 64, 0, 33, 99], 3000, 100, 4, 2, 128)
    gpu = on_gpu(t)
    call = lambda: ispa.attn_shared(**gpu, n_heads=4, n_kv_heads=2, max_q=max(counts))
    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = call()
    both = call()                                              # beside the one on the other stream
    torch.cuda.synchronize()
    for got in (again, both):
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    graphs, kept = [], []
    for _ in range(2):                                         # two graphs of the same tensors
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept.append(call())
        graphs.append(graph)
    for turn in range(3):                                      # lengths and rows are read on the device
        gpu["cache_lens"].copy_(torch.randint(0, 101, (6,), dtype=torch.int32, device=DEV))
        gpu["q"].copy_(torch.randn(gpu["q"].shape, device=DEV))
        want = call()
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for got in kept:
            assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]), turn


def test_distances_that_no_row_uses():
    # one request, one place, one prefix row: the distance to a next one does not exist and
    # may differ between keys and values
    t = make([3], [20], 40, 20, 2, 2, 64)
    gpu = on_gpu(t)
    want, want_lse = ispa.attn_shared(**gpu, n_heads=2)
    room = torch.zeros(4, 33, 128, dtype=BF16, device=DEV)
    room[2, :20] = gpu["k_cache"][0]
    out, lse = ispa.attn_shared(**{**gpu, "k_cache": room[2:3, :20]}, n_heads=2)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    t = make([2, 1], [1, 1], 1, 1, 2, 2, 64)
    gpu = on_gpu(t)
    both = torch.zeros(2, 5, 128, dtype=BF16, device=DEV)
    both[:, :1] = gpu["k_cache"]
    other = torch.zeros(2, 5 * 128, dtype=BF16, device=DEV)
    other[:, :128] = gpu["v_cache"][:, 0]
    prefix = torch.zeros(3, 256, dtype=BF16, device=DEV)
    prefix[0, :128] = gpu["k_prefix"][0]
    args = {**gpu, "k_cache": both[:, :1], "v_cache": other[:, :128].unsqueeze(1), "k_prefix": prefix[:, :128]}
    assert args["k_cache"].stride()[::2] == args["v_cache"].stride()[::2]
    out, lse = ispa.attn_shared(**args, n_heads=2, prefix_len=1)
    torch.cuda.synchronize()
    check(out, lse, exact(t, 2, 2))


def test_no_workspace_where_none_is_needed():
    # nobody has a key: no partial results, and no buffer for them
    L = ispa.lib()
    assert L.ispa_attn_shared_workspace_bytes(0, 0, 2, 3, 2, 2, 2, 64) == 0
    t = on_gpu(make([2, 1], [0, 0], 0, 0, 2, 2, 64))
    out, lse = torch.ones(3, 128, dtype=BF16, device=DEV), torch.ones(2, 3, device=DEV)
    st = L.ispa_attn_shared(t["q"].data_ptr(), 128, None, None, 0, 0, None, None, 0, 0, 0, t["q_start"].data_ptr(),
                            t["cache_lens"].data_ptr(), 2, 3, 2, 2, 2, 64, 0.0, out.data_ptr(), ispa.DTYPE_BF16, 128,
                            lse.data_ptr(), None, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == ispa.ISPA_OK and not out.any() and (lse == -math.inf).all()
