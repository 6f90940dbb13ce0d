"""The norm, rotary and shared-prefix entry points without a GPU: bad arguments are
refused before anything is enqueued (pointers here are fake and never read), and the
host-side frequencies follow their formulas."""

import ctypes
import math

import pytest
import torch

import paper_2607_00712_amd as ispa

E, U, OK = ispa.ISPA_ERR_INVALID_ARG, ispa.ISPA_ERR_UNSUPPORTED, ispa.ISPA_OK
BF16, F32 = ispa.DTYPE_BF16, ispa.DTYPE_F32


def call(name, defaults, **kw):
    assert set(kw) <= set(defaults), kw
    fn, types = getattr(ispa.lib(), name), ispa._SIGNATURES[name][1]
    values = list({**defaults, **kw}.values())
    assert len(values) == len(types)
    return fn(*[t(v or 0) if t is ctypes.c_void_p else v for t, v in zip(types, values)])


MB = 1 << 20
NORM = dict(x=MB, x_dtype=BF16, y=2 * MB, y_dtype=BF16, post=0, post_weight=0, gate=0, alpha=1.0, norm=1, weight=0,
            bias=0, scale=0, shift=0, rows=4, cols=64, group_rows=0, eps=1e-6, x_out=3 * MB, h=4 * MB, h_dtype=BF16,
            stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(x_dtype=2)), (U, dict(y_dtype=5)), (U, dict(h_dtype=-1)), (U, dict(norm=3)), (U, dict(post=-1)),
    (E, dict(cols=60)), (E, dict(cols=0)), (E, dict(cols=16392)), (E, dict(rows=-1)), (E, dict(rows=1 << 22)),
    (E, dict(eps=-1.0)), (E, dict(eps=math.nan)), (E, dict(eps=math.inf)), (E, dict(alpha=math.nan)),
    (E, dict(alpha=math.inf)), (E, dict(x=0)), (E, dict(x_out=0)), (E, dict(h=0)), (E, dict(x=MB + 8)),
    (E, dict(h=4 * MB + 2)), (E, dict(gate=MB * 5 + 4)),
    (E, dict(norm=0)),                                      # h without a norm
    (E, dict(norm=0, h=0, weight=5 * MB)),                  # weight without a norm
    (E, dict(norm=0, h=0, y=0)),                            # nothing to do
    (E, dict(y=0, gate=5 * MB)), (E, dict(y=0, post=1)), (E, dict(post_weight=5 * MB)),
    (E, dict(h=MB)), (E, dict(h=3 * MB + 16)), (E, dict(x_out=2 * MB)), (E, dict(x_out=MB + 16)),
    (E, dict(scale=4 * MB)),                                # h over scale
    (OK, dict(rows=0)),
])
def test_norm_residual_refusals(want, kw):
    assert call("ispa_norm_residual", NORM, **kw) == want


NORM_BACK = dict(d_h=MB, h_dtype=BF16, d_x_out=2 * MB, x_out=3 * MB, x_dtype=BF16, y=4 * MB, y_dtype=BF16, post=2,
                 post_weight=0, gate=0, alpha=1.0, norm=1, weight=0, bias=0, scale=0, rows=4, cols=64, group_rows=0,
                 eps=1e-6, d_x=5 * MB, d_y=6 * MB, d_gate=0, d_post_weight=0, d_weight=0, d_bias=0, d_scale=0, d_shift=0,
                 workspace=8 * MB, workspace_bytes=1 << 30, stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(x_dtype=3)), (U, dict(norm=4)), (E, dict(cols=12)), (E, dict(rows=-2)),
    (E, dict(d_h=0)), (E, dict(x_out=0)), (E, dict(d_x=0)), (E, dict(d_y=0)), (E, dict(y=0)),
    (E, dict(norm=0, d_h=0, x_out=0, d_x_out=0)), (E, dict(norm=0)),
    (E, dict(norm=0, d_h=0, x_out=0, d_weight=7 * MB)), (E, dict(y=0, d_y=0, post=0, d_gate=7 * MB)),
    (E, dict(post=0, d_post_weight=7 * MB)),
    (E, dict(d_x=3 * MB)), (E, dict(d_x=2 * MB + 16)), (E, dict(d_y=4 * MB)), (E, dict(d_y=5 * MB + 16)),
    (E, dict(d_gate=5 * MB)), (E, dict(d_gate=7 * MB, d_bias=7 * MB)), (E, dict(d_weight=7 * MB + 4)),
    (E, dict(d_gate=7 * MB, workspace=0)), (E, dict(d_gate=7 * MB, workspace=8 * MB + 128)),
    (E, dict(d_gate=7 * MB, workspace_bytes=64)), (E, dict(d_gate=8 * MB)),
    (OK, dict(rows=0)),
])
def test_norm_residual_backward_refusals(want, kw):
    assert call("ispa_norm_residual_backward", NORM_BACK, **kw) == want


def test_norm_workspace_sizes():
    f = ispa.lib().ispa_norm_residual_backward_workspace_bytes
    assert f(0, 64, 0) == 0 and f(4, 60, 0) == 0 and f(1 << 22, 64, 0) == 0
    for rows, cols, group in ((1, 8, 0), (4680, 1536, 1560), (4680, 1536, 1), (7, 16384, 3), (100, 64, 1000)):
        n = f(rows, cols, group)
        groups = -(-rows // (group or rows))
        assert n >= groups * 3 * cols * 4 and n % 256 == 0


PAIRS = (ctypes.c_int32 * 4)(3, 3, 2, 0)
ROT = dict(x=MB, x_dtype=BF16, ld_x=64, out=2 * MB, out_dtype=BF16, ld_out=64, positions=3 * MB, freqs=4 * MB,
           axis_pairs=PAIRS, n_axes=3, rotary_dim=16, interleaved=1, amplitude=1.0, inverse=0, rows=4, n_heads=2,
           head_dim=32, stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(x_dtype=2)), (U, dict(out_dtype=7)), (U, dict(head_dim=24)), (U, dict(head_dim=272, ld_x=544, ld_out=544)),
    (U, dict(rotary_dim=8)), (U, dict(rotary_dim=48)), (U, dict(rotary_dim=20)),
    (E, dict(n_axes=0)), (E, dict(n_axes=5)), (E, dict(n_axes=2)), (E, dict(axis_pairs=None)),
    (E, dict(rotary_dim=32)),                               # pairs do not add up
    (E, dict(axis_pairs=(ctypes.c_int32 * 4)(9, -3, 2, 0))),
    (E, dict(amplitude=math.nan)), (E, dict(rows=-1)), (E, dict(rows=1 << 30)), (E, dict(n_heads=0)),
    (E, dict(x=0)), (E, dict(out=0)), (E, dict(positions=0)), (E, dict(freqs=0)), (E, dict(x=MB + 8)),
    (E, dict(positions=3 * MB + 2)), (E, dict(freqs=4 * MB + 4)),
    (E, dict(ld_x=56)), (E, dict(ld_x=68)), (E, dict(ld_out=32)),
    (E, dict(out=MB + 16)), (E, dict(out=MB, ld_out=128)), (E, dict(out=MB, out_dtype=F32)), (E, dict(out=3 * MB)),
    (OK, dict(rows=0)),
])
def test_rotary_refusals(want, kw):
    assert call("ispa_rotary", ROT, **kw) == want


APPEND = dict(q=MB, ld_q=64, k=2 * MB, ld_k=32, v=3 * MB, ld_v=32, x_dtype=BF16, q_out=4 * MB, out_dtype=BF16,
              ld_out=64, k_cache=5 * MB, v_cache=6 * MB, cache_rows=100, slots=7 * MB, positions=8 * MB, freqs=9 * MB,
              axis_pairs=PAIRS, n_axes=3, rotary_dim=16, interleaved=1, amplitude=1.0, rows=4, n_heads=2, n_kv_heads=1,
              head_dim=32, stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(x_dtype=9)), (U, dict(head_dim=8)), (E, dict(n_kv_heads=0)), (E, dict(k=0)), (E, dict(v=0)),
    (E, dict(q_out=0)), (E, dict(k_cache=0)), (E, dict(slots=0)), (E, dict(slots=7 * MB + 4)), (E, dict(ld_k=24)),
    (E, dict(ld_v=36)), (E, dict(cache_rows=0)), (E, dict(cache_rows=1 << 62)), (E, dict(v_cache=5 * MB)),
    (E, dict(k_cache=2 * MB)), (E, dict(q_out=2 * MB)), (E, dict(q_out=5 * MB + 64)), (E, dict(q_out=MB, ld_out=72)),
    (E, dict(q_out=7 * MB)), (OK, dict(rows=0)),
])
def test_rotary_append_refusals(want, kw):
    assert call("ispa_rotary_append", APPEND, **kw) == want


@pytest.mark.parametrize("kw", [
    dict(q_out=MB + 128, ld_out=64, ld_q=64),               # q's own rows, the second head
    dict(q_out=MB + 2 * 96, ld_out=96, ld_q=96, k=MB + 2 * 64, ld_k=96),   # over q one row down, beside k
    dict(q_out=MB, ld_out=96, ld_q=96, k=MB + 2 * 56, ld_k=96),            # in place, but k begins inside
    dict(q_out=MB, ld_out=96, ld_q=96, k=MB + 2 * 72, ld_k=96),            # k runs into the next row
    dict(q_out=MB, ld_out=64, k=MB + 2 * 64, ld_k=96),                     # other distances
    dict(q_out=MB, ld_out=96, ld_q=96, v=MB + 2 * 32, ld_v=96),
    dict(rows=1 << 24),
])
def test_rotary_append_refuses_overlapping_columns(kw):
    assert call("ispa_rotary_append", APPEND, **kw) == E


SLOT = dict(q_start=MB, before=2 * MB, n_req=3, n_rows=10, capacity=20, sink=0, window=0, first_position=0,
            slots=3 * MB, positions=4 * MB, lens=5 * MB, stream=0)


@pytest.mark.parametrize("kw", [
    dict(q_start=0), dict(before=0), dict(lens=0), dict(slots=0), dict(positions=0), dict(n_req=0), dict(n_rows=-1),
    dict(capacity=0), dict(sink=-1, window=21), dict(sink=3), dict(sink=3, window=16), dict(window=-5), dict(window=19),
    dict(slots=3 * MB + 4), dict(lens=2 * MB), dict(positions=3 * MB), dict(lens=MB + 4),
])
def test_slot_map_refusals(kw):
    assert call("ispa_slot_map", SLOT, **kw) == E


SHARED = dict(q=MB, ld_q=128, k_prefix=2 * MB, v_prefix=3 * MB, prefix_len=100, ld_prefix=64, k_cache=4 * MB,
              v_cache=5 * MB, capacity=10, ld_cache=64, ld_request=640, q_start=6 * MB, cache_lens=7 * MB, n_req=3,
              n_rows=8, max_q=4, n_heads=2, n_kv_heads=1, head_dim=64, scale=0.0, out=8 * MB, out_dtype=BF16, ld_out=128,
              lse=9 * MB, workspace=16 * MB, workspace_bytes=1 << 30, stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(head_dim=96)), (U, dict(out_dtype=4)), (E, dict(n_kv_heads=3)), (E, dict(n_kv_heads=0)),
    (E, dict(prefix_len=-1)), (E, dict(prefix_len=1 << 31)), (E, dict(capacity=-1)), (E, dict(capacity=1 << 31)),
    (E, dict(n_req=0)), (E, dict(n_rows=-1)), (E, dict(max_q=0)), (E, dict(scale=math.nan)), (E, dict(scale=math.inf)),
    (E, dict(n_rows=1 << 26)), (E, dict(q=0)), (E, dict(out=0)), (E, dict(q_start=0)), (E, dict(cache_lens=0)),
    (E, dict(k_prefix=0)), (E, dict(v_cache=0)), (E, dict(q=MB + 8)), (E, dict(lse=9 * MB + 2)),
    (E, dict(k_cache=4 * MB + 2)), (E, dict(ld_q=64)), (E, dict(ld_q=132)), (E, dict(ld_prefix=56)),
    (E, dict(ld_cache=60)), (E, dict(ld_request=-640)), (E, dict(ld_request=644)), (E, dict(ld_out=120)),
    (E, dict(workspace=0)), (E, dict(workspace=16 * MB + 64)), (E, dict(workspace_bytes=512)), (E, dict(out=MB)),
    (E, dict(out=5 * MB)), (E, dict(lse=8 * MB)), (E, dict(workspace=2 * MB)), (E, dict(lse=16 * MB)),
    (OK, dict(n_rows=0)),
])
def test_attn_shared_refusals(want, kw):
    assert call("ispa_attn_shared", SHARED, **kw) == want


def test_attn_shared_workspace_sizes():
    f = ispa.lib().ispa_attn_shared_workspace_bytes
    assert f(100, 10, 3, 0, 1, 2, 1, 64) == 0 and f(100, 10, 3, 8, 1, 2, 1, 96) == 0 and f(100, 10, 0, 8, 1, 2, 1, 64) == 0
    for size in ((0, 0, 1, 1, 1, 1, 1, 64), (32760, 1024, 64, 64, 1, 12, 12, 128), (1, 1, 4, 6240, 1560, 32, 4, 128),
                 (0x7fffffff, 0x7fffffff, 1, 1, 1, 1, 1, 64)):
        splits_at_least = (size[0] > 0) + (size[1] > 0)
        assert f(*size) >= splits_at_least * size[3] * size[5] * (size[7] + 1) * 4 and f(*size) % 256 == 0


def frequencies(axis_pairs, **kw):
    freqs, amplitude = ispa.rotary_frequencies(axis_pairs, device="cpu", **kw)
    assert freqs.dtype == torch.float64
    return freqs.tolist(), amplitude


def test_rotary_frequencies():
    f, a = frequencies(64, base=5e5)
    assert a == 1.0 and f == pytest.approx([5e5 ** (-j / 64) for j in range(64)], rel=1e-14)
    f, _ = frequencies((22, 21, 21))
    assert f == pytest.approx([1e4 ** (-j / n) for n in (22, 21, 21) for j in range(n)], rel=1e-14)
    f, _ = frequencies(32, scaling="linear", factor=4.0)
    assert f == pytest.approx([1e4 ** (-j / 32) / 4 for j in range(32)], rel=1e-14)
    f, _ = frequencies(32, scaling="base", factor=8.0)
    g, _ = frequencies(32)
    assert f[0] == 1.0 and f[-1] == pytest.approx(g[-1] / 8, rel=1e-13)
    f, a = frequencies(64, scaling="parts", factor=16.0, original_length=4096)
    assert a == pytest.approx(0.1 * math.log(16) + 1)
    g, _ = frequencies(64)
    turns = [4096 * x / (2 * math.pi) for x in g]
    for x, y, t in zip(f, g, turns):
        assert y / 16 * (1 - 1e-12) <= x <= y
        if t > 32 * 1.2:
            assert x == pytest.approx(y, rel=1e-14)
        if t < 1 / 1.2:
            assert x == pytest.approx(y / 16, rel=1e-14)


@pytest.mark.parametrize("pairs, kw", [
    ((), {}), ((0,), {}), ((129,), {}), ((64, 65), {}), ((1, 1, 1, 1, 1), {}), (8, dict(base=1.0)),
    (8, dict(base=math.inf)), (8, dict(scaling="linear", factor=0.5)), (8, dict(scaling="parts", factor=2.0)),
    ((8, 8), dict(scaling="parts", factor=2.0, original_length=100)),
    (8, dict(scaling="parts", factor=2.0, original_length=100, beta_fast=1.0, beta_slow=2.0)),
])
def test_rotary_frequencies_refusals(pairs, kw):
    with pytest.raises(ispa.IspaError):
        ispa.rotary_frequencies(pairs, device="cpu", **kw)


def test_binding_refuses_host_tensors_and_names():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    i32 = torch.zeros(4, dtype=torch.int32)
    f = torch.ones(8, dtype=torch.float64)
    for fn in (lambda: ispa.norm_residual(x), lambda: ispa.norm_residual(x, norm="batch"),
               lambda: ispa.norm_residual_backward(x, x), lambda: ispa.rotary(x, i32, f, 2),
               lambda: ispa.slot_map(i32, i32[:3], 4, 4), lambda: ispa.rotary_append(x, x, x, i32, i32.long(), f, 2, x, x),
               lambda: ispa.attn_shared(x, x, x, x[None], x[None], i32[:2], i32[:1], 1),
               lambda: ispa.rotary_frequencies(8, scaling="other")):
        with pytest.raises(ValueError):
            fn()
    with pytest.raises(TypeError):
        ispa.norm_residual(x.double())


@pytest.mark.parametrize("want, kw", [
    (E, dict(n_real=10 * MB + 2)), (E, dict(q_out=10 * MB)), (E, dict(n_real=4 * MB + 252)), (E, dict(k_cache=10 * MB - 64)),
    (E, dict(v_cache=10 * MB)), (E, dict(slots=0)), (E, dict(q=0)), (U, dict(head_dim=8)), (E, dict(q_out=2 * MB)),
    (E, dict(rows=-1)), (OK, dict(rows=0)), (OK, dict(rows=0, n_real=0)),
])
def test_rotary_append_batch_refusals(want, kw):
    args = {}
    for name, value in APPEND.items():
        args[name] = value
        if name == "slots":
            args["n_real"] = 10 * MB
    assert call("ispa_rotary_append_batch", args, **kw) == want


@pytest.mark.parametrize("pairs", [16, 64, 1])
@pytest.mark.parametrize("length", [3.0, 40.0, 4096.0, 54000.0, 65536.0, 131072.0, 1e6, 1e8])
@pytest.mark.parametrize("factor", [4.0, 16.0])
def test_rotary_frequencies_in_parts(pairs, length, factor):
    # trained lengths around 2 pi base: the ramp ends behind the last pair there, and lies
    # behind it whole further on. The pair (not whole) that turns beta times in `length` is
    # pairs ln(length / (2 pi beta)) / ln(base); the ramp runs between the whole ones around
    # those of beta_fast and beta_slow, from the first pair on at the least
    f, _ = frequencies(pairs, scaling="parts", factor=factor, original_length=length)
    at = lambda beta: pairs * math.log(length / (2 * math.pi * beta)) / math.log(1e4)
    lo, hi = max(0, math.floor(at(32.0))), math.ceil(at(1.0))
    for j, x in enumerate(f):
        y = 1e4 ** (-j / pairs)
        turns = length * y / (2 * math.pi)
        if turns > 32:
            assert x == pytest.approx(y, rel=1e-13), j
        elif turns < 1:
            assert x == pytest.approx(y / factor, rel=1e-13), j
        else:
            ramp = min(1.0, max(0.0, (j - lo) / (hi - lo))) if hi > lo else 1.0
            assert x == pytest.approx(y * (1 - ramp) + y / factor * ramp, rel=1e-12), j


def test_rotary_frequencies_of_long_trained_lengths():
    # 64 pairs, base 1e4, trained to 131072: the slowest pair turns 2.4 times there, more than
    # beta_slow. Its place is 63 on a ramp from 45 to 70: 18 / 25 of the way to a quarter.
    f, _ = frequencies(64, scaling="parts", factor=4.0, original_length=131072)
    y = 1e4 ** (-63 / 64)
    assert f[63] / y == pytest.approx(1 - 18 / 25 * 0.75, rel=1e-12)
