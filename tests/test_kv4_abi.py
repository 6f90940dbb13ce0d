"""The entry points of heads' norms and of the 4-bit cache without a GPU: bad arguments are
refused before anything is enqueued (pointers here are fake and never read), and the sizes
follow their formulas."""

import ctypes
import math

import pytest
import torch

import paper_2607_00712_amd as ispa
from kv4_format import NUMBERS, decode, encode, pack, unpack
from test_operators_abi import call

E, U, OK = ispa.ISPA_ERR_INVALID_ARG, ispa.ISPA_ERR_UNSUPPORTED, ispa.ISPA_OK
BF16, F32 = ispa.DTYPE_BF16, ispa.DTYPE_F32
MB = 1 << 20
PAIRS = (ctypes.c_int32 * 4)(3, 3, 2, 0)

TURN = dict(q=MB, ld_q=64, k=2 * MB, ld_k=32, x_dtype=BF16, norm=2, q_weight=0, k_weight=0, q_bias=0, k_bias=0, eps=1e-6,
            q_out=3 * MB, ld_qo=64, k_out=4 * MB, ld_ko=32, out_dtype=BF16, positions=5 * MB, freqs=6 * MB,
            axis_pairs=PAIRS, n_axes=3, rotary_dim=16, interleaved=1, amplitude=1.0, rows=4, n_heads=2, n_kv_heads=1,
            head_dim=32, stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(x_dtype=2)), (U, dict(out_dtype=7)), (U, dict(norm=0)), (U, dict(norm=3)), (U, dict(head_dim=24)),
    (U, dict(rotary_dim=8)), (U, dict(rotary_dim=48)), (E, dict(rotary_dim=32)), (E, dict(n_axes=0)), (E, dict(n_axes=2)),
    (E, dict(eps=-1.0)), (E, dict(eps=math.nan)), (E, dict(eps=math.inf)), (E, dict(amplitude=math.inf)),
    (E, dict(rows=-1)), (E, dict(rows=1 << 24)), (E, dict(n_heads=0)), (E, dict(n_kv_heads=0)),
    (E, dict(q=0)), (E, dict(q_out=0)), (E, dict(k_out=0)), (E, dict(k=0)), (E, dict(k=0, k_out=0, k_weight=7 * MB)),
    (E, dict(q=MB + 8)), (E, dict(k_weight=7 * MB + 4)), (E, dict(ld_q=56)), (E, dict(ld_q=68)), (E, dict(ld_ko=24)),
    (E, dict(q_out=MB + 16)), (E, dict(q_out=MB, ld_qo=128)), (E, dict(q_out=MB, out_dtype=F32)), (E, dict(k_out=3 * MB)),
    (E, dict(q_out=2 * MB)), (E, dict(q_out=5 * MB)), (E, dict(k_out=MB)), (E, dict(q_weight=3 * MB)),
    (E, dict(q_bias=4 * MB)), (E, dict(freqs=3 * MB)),
    (OK, dict(rows=0)), (OK, dict(rows=0, k=0, k_out=0)),
])
def test_norm_rotary_refusals(want, kw):
    assert call("ispa_norm_rotary", TURN, **kw) == want


BACK = dict(d_q_out=MB, ld_gq=64, d_k_out=2 * MB, ld_gk=32, g_dtype=BF16, q=3 * MB, ld_q=64, k=4 * MB, ld_k=32,
            x_dtype=BF16, norm=2, q_weight=0, k_weight=0, eps=1e-6, d_q=5 * MB, ld_dq=64, d_k=6 * MB, ld_dk=32,
            d_q_weight=0, d_k_weight=0, d_q_bias=0, d_k_bias=0, positions=7 * MB, freqs=8 * MB, axis_pairs=PAIRS,
            n_axes=3, rotary_dim=16, interleaved=1, amplitude=1.0, rows=4, n_heads=2, n_kv_heads=1, head_dim=32,
            workspace=9 * MB, workspace_bytes=1 << 20, stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(g_dtype=3)), (U, dict(norm=0)), (U, dict(x_dtype=-1)), (E, dict(d_q_out=0)), (E, dict(d_k_out=0)),
    (E, dict(q=0)), (E, dict(k=0)), (E, dict(d_q=0)), (E, dict(d_k=0)), (E, dict(eps=-0.5)),
    (E, dict(k=0, d_k_out=0, d_k=0, d_k_bias=10 * MB)), (E, dict(ld_gq=32)), (E, dict(ld_dk=36)),
    (E, dict(d_q=3 * MB)), (E, dict(d_q=4 * MB)), (E, dict(d_q=2 * MB)), (E, dict(d_q=MB, g_dtype=F32)),
    (E, dict(d_k=5 * MB)), (E, dict(d_q=7 * MB)), (E, dict(d_q_weight=5 * MB)), (E, dict(d_q_weight=9 * MB)),
    (E, dict(d_q_weight=10 * MB, d_k_bias=10 * MB)), (E, dict(d_q_weight=10 * MB + 4)),
    (E, dict(d_q_weight=10 * MB, workspace=0)), (E, dict(d_q_weight=10 * MB, workspace=9 * MB + 128)),
    (E, dict(d_q_weight=10 * MB, workspace_bytes=64)), (E, dict(d_k_weight=10 * MB, k_weight=10 * MB)),
    (OK, dict(rows=0)),
])
def test_norm_rotary_backward_refusals(want, kw):
    assert call("ispa_norm_rotary_backward", BACK, **kw) == want


APPEND = dict(q=MB, ld_q=128, k=2 * MB, ld_k=64, v=3 * MB, ld_v=64, x_dtype=BF16, norm=0, q_weight=0, k_weight=0, q_bias=0,
              k_bias=0, eps=1e-6, q_out=4 * MB, out_dtype=BF16, ld_out=128, cache=5 * MB, n_pages=8, page_size=32,
              page_table=6 * MB, n_req=2, max_pages=4, slots=7 * MB, n_real=0, positions=8 * MB, freqs=9 * MB,
              axis_pairs=PAIRS, n_axes=3, rotary_dim=16, interleaved=1, amplitude=1.0, rows=4, n_heads=2, n_kv_heads=1,
              head_dim=64, stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(x_dtype=9)), (U, dict(head_dim=32)), (U, dict(head_dim=96, ld_q=192, ld_k=96, ld_v=96, ld_out=192)),
    (U, dict(norm=5)), (E, dict(q_weight=10 * MB)), (E, dict(norm=2, eps=-1.0)),
    (E, dict(page_size=16)), (E, dict(page_size=48)), (E, dict(page_size=1 << 17)), (E, dict(page_size=0)),
    (E, dict(n_pages=0)), (E, dict(n_pages=1 << 32)), (E, dict(n_req=0)), (E, dict(max_pages=0)),
    (E, dict(max_pages=1 << 26)), (E, dict(cache=0)), (E, dict(cache=5 * MB + 8)), (E, dict(page_table=0)),
    (E, dict(page_table=6 * MB + 2)), (E, dict(q=0)), (E, dict(k=0)), (E, dict(v=0)), (E, dict(q_out=0)),
    (E, dict(slots=0)), (E, dict(slots=7 * MB + 4)), (E, dict(n_real=7 * MB + 2)), (E, dict(positions=0)),
    (E, dict(n_kv_heads=0)), (E, dict(ld_v=56)), (E, dict(q_out=2 * MB)), (E, dict(q_out=MB + 64)),
    (E, dict(cache=MB)), (E, dict(cache=6 * MB)), (E, dict(cache=4 * MB - 16)), (E, dict(slots=5 * MB + 64)),
    (E, dict(n_real=4 * MB)), (E, dict(norm=1, k_weight=5 * MB + 16)),
    (OK, dict(rows=0)),
])
def test_append_refusals(want, kw):
    assert call("ispa_kv4_append", APPEND, **kw) == want


READ = dict(cache=MB, n_pages=8, page_size=32, page_table=2 * MB, n_req=2, max_pages=4, slots=3 * MB, rows=4, n_kv_heads=1,
            head_dim=64, k=4 * MB, v=5 * MB, out_dtype=BF16, stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(head_dim=48)), (U, dict(out_dtype=2)), (E, dict(page_size=33)), (E, dict(cache=0)), (E, dict(slots=0)),
    (E, dict(k=0)), (E, dict(v=0)), (E, dict(k=4 * MB + 8)), (E, dict(rows=-1)), (E, dict(rows=1 << 28)),
    (E, dict(k=5 * MB)), (E, dict(k=MB)), (E, dict(v=2 * MB)), (E, dict(v=3 * MB)), (OK, dict(rows=0)),
])
def test_read_refusals(want, kw):
    assert call("ispa_kv4_read", READ, **kw) == want


ATTN = dict(q=MB, ld_q=128, cache=2 * MB, n_pages=8, page_size=32, page_table=3 * MB, max_pages=4, q_start=4 * MB,
            cache_lens=5 * MB, n_req=2, n_rows=4, max_q=2, n_heads=2, n_kv_heads=1, head_dim=64, scale=0.0, out=6 * MB,
            out_dtype=BF16, ld_out=128, lse=0, workspace=8 * MB, workspace_bytes=1 << 30, stream=0)


@pytest.mark.parametrize("want, kw", [
    (U, dict(head_dim=32)), (U, dict(out_dtype=3)), (E, dict(page_size=40)), (E, dict(max_pages=0)), (E, dict(n_req=0)),
    (E, dict(n_rows=-1)), (E, dict(n_rows=1 << 26)), (E, dict(max_q=0)), (E, dict(n_heads=3, n_kv_heads=2)),
    (E, dict(n_heads=0)), (E, dict(scale=math.nan)), (E, dict(scale=math.inf)), (E, dict(q=0)), (E, dict(out=0)),
    (E, dict(q_start=0)), (E, dict(cache_lens=0)), (E, dict(cache=0)), (E, dict(page_table=0)), (E, dict(q=MB + 8)),
    (E, dict(lse=7 * MB + 2)), (E, dict(ld_q=120)), (E, dict(ld_out=100)), (E, dict(workspace=0)),
    (E, dict(workspace=8 * MB + 16)), (E, dict(workspace_bytes=16)), (E, dict(out=MB)), (E, dict(out=2 * MB)),
    (E, dict(out=3 * MB)), (E, dict(lse=6 * MB)), (E, dict(lse=MB)), (E, dict(workspace=2 * MB)), (E, dict(out=8 * MB)),
    (OK, dict(n_rows=0)),
])
def test_attention_refusals(want, kw):
    assert call("ispa_attn_kv4", ATTN, **kw) == want


def test_sizes():
    L = ispa.lib()
    assert [L.ispa_kv4_page_bytes(p, d) for p, d in ((32, 64), (64, 128), (65536, 128))] == [32 * 68, 64 * 136, 65536 * 136]
    assert not any(L.ispa_kv4_page_bytes(p, d) for p, d in ((16, 64), (96, 64), (1 << 17, 64), (32, 32), (0, 64)))
    f = L.ispa_norm_rotary_backward_workspace_bytes
    assert f(0, 1, 1, 64) == 0 and f(4, 1, 1, 24) == 0 and f(4, 0, 1, 64) == 0 and f(1 << 24, 1, 1, 64) == 0
    for rows, heads, kv, d in ((1, 1, 0, 16), (4680, 40, 40, 128), (7, 32, 1, 256), (1 << 23, 1, 1, 16)):
        n = f(rows, heads, kv, d)
        assert n >= (1 + (kv > 0)) * 2 * d * 4 and n % 256 == 0 and n <= 2 * 1024 * 2 * d * 4
    f = L.ispa_attn_kv4_workspace_bytes
    assert f(32, 4, 2, 0, 1, 2, 1, 64) == 0 and f(48, 4, 2, 4, 1, 2, 1, 64) == 0 and f(32, 4, 2, 4, 1, 2, 1, 96) == 0
    # bounded by the device's runs, whatever the lengths, and small where there are few units
    assert 0 < f(32, 1, 1, 1, 1, 1, 1, 64) < f(64, 4096, 64, 64, 1, 32, 8, 128) <= 64 << 20
    assert f(64, 4096, 64, 64, 1, 32, 8, 128) == f(64, 1 << 20, 64, 64, 1, 32, 8, 128)


def test_format_helpers():
    """The tests' own format: every number is held, rounding is to the nearest: a step
    is one power up to 2 above 4 powers, so half of it is at most one fifth of a largest value of 5
    powers (one above 4 and below 5 rounds to 4, off by less)."""
    g = torch.Generator().manual_seed(0)
    x = NUMBERS[torch.randint(0, 16, (4, 2, 32, 64), generator=g)]
    x[..., ::32] = 6.0  # (each block has its largest number)
    codes, powers = encode(x * 0.25)
    assert torch.equal(decode(codes, powers), x * 0.25) and (powers == 125).all()
    (a, b), (c, d) = unpack(pack((codes, powers), (codes.flip(2), powers)), 64)
    assert torch.equal(a, codes) and torch.equal(b, powers) and torch.equal(c, codes.flip(2)) and torch.equal(d, powers)
    y = torch.randn(50, 64, generator=g, dtype=torch.float64)
    codes, powers = encode(y)
    top = y.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True).expand(-1, -1, 32).flatten(1)
    assert ((decode(codes, powers) - y).abs() <= top / 5).all()
