"""Rotary positions, slot maps and the append into caches on the GPU against their
definitions in 64 bits.

Tolerance of a turned value: its rounding, |value| eps(dtype) / 2, and the error of cos
and sin: the fraction of a turn is rounded to fp32 (half a step of at most one half
turn: pi 2^-24 in the angle), sincospi is within 2 steps (2^-23), the products and the
sum round three times (3 x 2^-24): together below 2^-21 of |a| + |b|, times the
amplitude.
"""

import pytest
import torch

import paper_2607_00712_amd as ispa

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def turned(x, positions, freqs, axes, head_dim, interleaved, amplitude, inverse=False):
    """x [rows, heads * head_dim] turned in 64 bits, and the tolerance's magnitudes."""
    half = len(freqs)
    axis = torch.tensor([k for k, n in enumerate(axes) for _ in range(n)])
    angle = positions.double().view(len(x), -1)[:, axis] * freqs
    c, s = angle.cos()[:, None] * amplitude, angle.sin()[:, None] * amplitude * (-1 if inverse else 1)
    x = x.double().view(len(x), -1, head_dim)
    out, size = x.clone(), torch.zeros_like(x)
    first = torch.arange(half)
    i, k = (2 * first, 2 * first + 1) if interleaved else (first, first + half)
    a, b = x[..., i], x[..., k]
    out[..., i], out[..., k] = a * c - b * s, a * s + b * c
    size[..., i] = size[..., k] = (a.abs() + b.abs()) * abs(amplitude)
    return out.flatten(1), size.flatten(1)


def check(got, want, size, what):
    tol = want.abs() * (torch.finfo(got.dtype).eps / 2) + size * 2.0 ** -21
    err = (got.double().cpu() - want).abs()
    assert torch.all(err <= tol), f"{what}: {(err - tol).max().item():.3e} over the tolerance"


CASES = [
    # rows, heads, head_dim, axes, interleaved, amplitude, dtype, far
    (1, 1, 16, (8,), True, 1.0, F32, 1), (3, 2, 64, (32,), False, 1.2, BF16, 1), (5, 3, 64, (16,), False, 1.0, F32, 1),
    (5, 3, 64, (16,), True, 1.0, BF16, 1), (7, 12, 128, (22, 21, 21), True, 1.0, BF16, 1),
    (7, 12, 128, (22, 21, 21), False, 1.0, F32, 1), (33, 5, 48, (8, 16), True, 0.5, F32, 1),
    (2, 40, 256, (32, 32, 32, 32), False, 1.0, BF16, 1), (2050, 2, 64, (32,), True, 1.0, BF16, 1),
    (4099, 1, 128, (64,), False, 1.0, BF16, 1), (9, 2, 128, (64,), True, 1.0, F32, 2000003),
    (9, 2, 128, (64,), False, 1.0, F32, 2 ** 31 - 40), (4, 300, 64, (32,), True, 1.0, F32, -5000),
    # eight tokens to a workgroup, the last ones fewer
    (8195, 1, 48, (8, 16), True, 0.5, BF16, 1), (8200, 2, 80, (24,), False, 1.0, F32, 1),
]


def inputs(rows, heads, head_dim, axes, dtype, far):
    g = torch.Generator().manual_seed(rows + heads)
    x = torch.randn(rows, heads * head_dim, generator=g).to(dtype)
    p = torch.randint(0, 37, (rows, len(axes)), generator=g, dtype=torch.int32)
    p += (torch.randint(0, 3, (rows, len(axes)), generator=g, dtype=torch.int32) * (far // 3)) if far != 1 else 0
    freqs, _ = ispa.rotary_frequencies(axes, device="cpu")
    return x, p, freqs


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_rotary(case, inverse):
    rows, heads, head_dim, axes, interleaved, amplitude, dtype, far = CASES[case]
    x, p, f = inputs(rows, heads, head_dim, axes, dtype, far)
    print(f"rotary {CASES[case]}", flush=True)
    got = ispa.rotary(x.to(DEV), p.to(DEV), f.to(DEV), heads, axes=axes, interleaved=interleaved, amplitude=amplitude,
                      inverse=inverse)
    torch.cuda.synchronize()
    want, size = turned(x, p, f, axes, head_dim, interleaved, amplitude, inverse)
    check(got, want, size, "rotary")
    # values behind the turned part pass through bit for bit
    part = 2 * len(f)
    assert torch.equal(got.cpu().view(rows, heads, head_dim)[..., part:], x.view(rows, heads, head_dim)[..., part:])


def test_rotary_strides_types_and_in_place():
    x, p, f = inputs(21, 4, 64, (32,), BF16, 1)
    want = ispa.rotary(x.to(DEV), p.to(DEV), f.to(DEV), 4)
    wide = torch.full((21, 3 * 256), 7.0, dtype=BF16, device=DEV)
    wide[:, 256:512] = x.to(DEV)
    out = torch.full((21, 512), 5.0, dtype=BF16, device=DEV)
    ispa.rotary(wide[:, 256:512], p.to(DEV), f.to(DEV), 4, out=out[:, :256])
    assert torch.equal(out[:, :256], want) and (out[:, 256:] == 5).all()
    ispa.rotary(wide[:, 256:512], p.to(DEV), f.to(DEV), 4, out=wide[:, 256:512])
    assert torch.equal(wide[:, 256:512], want) and (wide[:, :256] == 7).all() and (wide[:, 512:] == 7).all()
    as_f32 = ispa.rotary(x.to(DEV), p.to(DEV), f.to(DEV), 4, out=torch.empty(21, 256, device=DEV))
    assert torch.equal(as_f32.to(BF16), want)
    one = ispa.rotary(x.to(DEV), p[:, 0].to(DEV).contiguous(), f.to(DEV), 4)
    assert torch.equal(one, want)
    assert ispa.rotary(x[:0].to(DEV), p[:0].to(DEV), f.to(DEV), 4).shape == (0, 256)
    for bad in (lambda: ispa.rotary(x.to(DEV).t(), p.to(DEV), f.to(DEV), 4),
                lambda: ispa.rotary(x.to(DEV), p.to(DEV), f.to(DEV), 4, axes=(16, 15)),
                lambda: ispa.rotary(x.to(DEV), p[:5].to(DEV), f.to(DEV), 4),
                lambda: ispa.rotary(x.to(DEV)[:, :252], p.to(DEV), f.to(DEV), 4),
                lambda: ispa.rotary(x.to(DEV).expand(21, 256)[:1].expand(21, 256), p.to(DEV), f.to(DEV), 4)):
        with pytest.raises(ValueError):
            bad()
    y = wide[:, :512]
    with pytest.raises(ispa.IspaError):                     # overlapping, not in place
        ispa.rotary(y[:, :256], p.to(DEV), f.to(DEV), 4, out=y[:, 128:384])


def test_inverse_is_the_transpose():
    # <rotary(x), y> = <x, rotary(y, inverse)>: fp32 products of 256 values, 2^-21 each
    x, p, f = inputs(16, 4, 64, (32,), F32, 1)
    y = torch.randn(16, 256, generator=torch.Generator().manual_seed(9))
    a = ispa.rotary(x.to(DEV), p.to(DEV), f.to(DEV), 4, amplitude=1.3).double().cpu()
    b = ispa.rotary(y.to(DEV), p.to(DEV), f.to(DEV), 4, amplitude=1.3, inverse=True).double().cpu()
    left, right = (a * y.double()).sum(1), (x.double() * b).sum(1)
    assert torch.all((left - right).abs() <= 2.0 ** -20 * 1.3 * 2 * (x.double().abs().sum(1) * y.abs().max(1)[0]))


def slots_of(starts, before, capacity, rows, sink, window, first):
    slots, positions = [-1] * rows, [0] * rows
    lens = []
    for b, at in enumerate(before):
        m = starts[b + 1] - starts[b]
        lens.append(at + m)
        for i in range(m):
            t = at + i
            positions[starts[b] + i] = first + t
            place = t
            if window and t >= sink:
                place = sink + (t - sink) % window if m - i <= window else -1
            if 0 <= place < capacity:
                slots[starts[b] + i] = b * capacity + place
    return slots, positions, lens


@pytest.mark.parametrize("counts, before, capacity, pad, sink, window, first", [
    ([1], [0], 1, 0, 0, 0, 0), ([3, 0, 2, 1], [5, 9, 0, 7], 10, 4, 0, 0, 100), ([0, 0], [1, 2], 4, 3, 0, 0, 0),
    ([4, 5], [8, 10], 10, 0, 0, 0, 0),                       # not all of them fit
    ([7, 2, 30], [0, 100, 3], 12, 2, 4, 8, 0), ([5, 9], [0, 1], 6, 0, 0, 6, 0), ([3], [7], 5, 1, 4, 1, 0),
    ([1] * 300, list(range(300)), 400, 5, 0, 0, 7), ([2, 1, 0] * 1500, [3] * 4500, 9, 0, 0, 0, 0),
    ([70000, 1, 70001], [0, 5, 9], 80000, 3, 1000, 79000, 1 << 20),
])
def test_slot_map(counts, before, capacity, pad, sink, window, first):
    starts = [0]
    for m in counts:
        starts.append(starts[-1] + m)
    rows = starts[-1] + pad
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    slots, positions, lens = ispa.slot_map(i32(starts), i32(before), capacity, rows, sink, window, first)
    want = slots_of(starts, before, capacity, rows, sink, window, first)
    assert slots.dtype == torch.int64 and positions.dtype == torch.int32 and lens.dtype == torch.int32
    assert slots.tolist() == want[0] and positions.tolist() == want[1] and lens.tolist() == want[2]
    kept = [s for s in want[0] if s >= 0]
    assert len(set(kept)) == len(kept)


def test_slot_map_ring_is_local_kv():
    # the places are those that LocalKV's ring takes for the same sequence of appends
    sink, window, hidden = 3, 10, 8
    tokens = torch.arange(60, dtype=F32, device=DEV)[:, None].expand(60, hidden).to(BF16).contiguous()
    kv = ispa.LocalKV(tokens[:5].contiguous(), tokens[:5].contiguous(), 5, window, sink)
    ring = torch.zeros(sink + window, hidden, dtype=BF16, device=DEV)
    ring[:5] = tokens[:5]
    at = 5
    for m in (1, 4, 13, 2, 30):
        new = tokens[at:at + m].contiguous()
        kv.append(new, new)
        slots, _, lens = ispa.slot_map(torch.tensor([0, m], dtype=torch.int32, device=DEV),
                                       torch.tensor([at], dtype=torch.int32, device=DEV), sink + window, m, sink, window)
        ring[slots[slots >= 0]] = new[slots >= 0]
        at += m
        assert lens.item() == at and torch.equal(ring[:kv.rows], kv.k[:kv.rows])


@pytest.mark.parametrize("dtype, out_dtype", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("heads, kv_heads, head_dim, axes, interleaved", [
    (4, 4, 64, (32,), True), (12, 3, 128, (22, 21, 21), True), (8, 1, 128, (32,), False), (2, 5, 16, (8,), False),
    (40, 40, 32, (16,), True),
])
def test_rotary_append(heads, kv_heads, head_dim, axes, interleaved, dtype, out_dtype):
    rows, capacity = 45, 13
    g = torch.Generator().manual_seed(heads)
    q = torch.randn(rows, heads * head_dim, generator=g).to(dtype)
    k, v = (torch.randn(rows, kv_heads * head_dim, generator=g).to(dtype) for _ in range(2))
    p = torch.randint(0, 100000, (rows, len(axes)), generator=g, dtype=torch.int32)
    f, _ = ispa.rotary_frequencies(axes, device="cpu")
    slots = torch.randperm(4 * capacity, generator=g)[:rows].clone()
    slots[[3, 20]] = -1
    slots[[5, 44]] = torch.tensor([4 * capacity, 1 << 40])     # behind the caches: left alone
    wide = torch.cat((q, k, v), 1).to(DEV)                      # one product's slices
    a, b = heads * head_dim, (heads + kv_heads) * head_dim
    caches = [torch.full((4, capacity, kv_heads * head_dim), 3.0, dtype=BF16, device=DEV) for _ in range(2)]
    out = torch.full((rows, a), 9.0, dtype=out_dtype, device=DEV)
    ret = ispa.rotary_append(wide[:, :a], wide[:, a:b], wide[:, b:], p.to(DEV), slots.to(DEV), f.to(DEV), heads, *caches,
                             n_kv_heads=kv_heads, axes=axes, interleaved=interleaved, amplitude=1.1, q_out=out)
    torch.cuda.synchronize()
    assert ret is out
    kept = (slots >= 0) & (slots < 4 * capacity)
    want, size = turned(q, p, f, axes, head_dim, interleaved, 1.1)
    check(out[kept], want[kept], size[kept], "q")
    assert (out.cpu()[~kept] == 9).all()
    want, size = turned(k, p, f, axes, head_dim, interleaved, 1.1)
    flat = [c.view(4 * capacity, -1).cpu() for c in caches]
    check(flat[0][slots[kept]], want[kept], size[kept], "k")
    assert torch.equal(flat[1][slots[kept]], v[kept].to(BF16))
    untouched = torch.ones(4 * capacity, dtype=torch.bool)
    untouched[slots[kept]] = False
    assert (flat[0][untouched] == 3).all() and (flat[1][untouched] == 3).all()


@pytest.mark.parametrize("rows", [1, 2, 21])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_and_turn_inside_one_wide_product(rows, dtype):
    # q turned in place between k and v of the same rows, and into other columns of them:
    # what is beside it stays as it was
    heads, kv_heads, head_dim = 6, 2, 64
    nq, nk = heads * head_dim, kv_heads * head_dim
    g = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, 2 * nq + 2 * nk, generator=g).to(dtype)
    p = torch.randint(0, 5000, (rows, 1), generator=g, dtype=torch.int32)
    f, _ = ispa.rotary_frequencies(32, device="cpu")
    wide = x.to(DEV)
    k, q, v, spare = wide.split((nk, nq, nk, nq), 1)
    caches = [torch.zeros(rows, nk, dtype=BF16, device=DEV) for _ in range(2)]
    slots = torch.arange(rows, device=DEV)
    assert ispa.rotary_append(q, k, v, p.to(DEV), slots, f.to(DEV), heads, *caches, n_kv_heads=kv_heads, q_out=q) is q
    want, size = turned(x[:, nk:nk + nq], p, f, (32,), head_dim, True, 1.0)
    check(q, want, size, "q")
    want, size = turned(x[:, :nk], p, f, (32,), head_dim, True, 1.0)
    check(caches[0], want, size, "k")
    assert torch.equal(caches[1].cpu(), x[:, nk + nq:2 * nk + nq].to(BF16))
    assert torch.equal(k.cpu(), x[:, :nk]) and torch.equal(wide[:, nk + nq:].cpu(), x[:, nk + nq:])
    before = wide.clone()
    ispa.rotary(q, p.to(DEV), f.to(DEV), heads, inverse=True, out=spare)
    want, size = turned(before[:, nk:nk + nq].cpu(), p, f, (32,), head_dim, True, 1.0, inverse=True)
    check(spare, want, size, "spare")
    assert torch.equal(wide[:, :2 * nk + nq], before[:, :2 * nk + nq])


def test_append_of_many_rows():
    # several tokens to a workgroup, rows without a slot among them, a head of 80 values of
    # which 48 turn
    rows, heads, kv_heads, head_dim = 8203, 3, 1, 80
    g = torch.Generator().manual_seed(8)
    q, k, v = (torch.randn(rows, n * head_dim, generator=g).to(BF16) for n in (heads, kv_heads, kv_heads))
    p = torch.randint(0, 100000, (rows, 1), generator=g, dtype=torch.int32)
    f, _ = ispa.rotary_frequencies(24, device="cpu")
    slots = torch.randperm(9000, generator=g)[:rows].clone()
    slots[torch.randperm(rows, generator=g)[:700]] = -1
    caches = [torch.full((9000, head_dim), 3.0, dtype=BF16, device=DEV) for _ in range(2)]
    out = torch.full((rows, heads * head_dim), 9.0, dtype=BF16, device=DEV)
    ispa.rotary_append(q.to(DEV), k.to(DEV), v.to(DEV), p.to(DEV), slots.to(DEV), f.to(DEV), heads, *caches,
                       n_kv_heads=kv_heads, interleaved=False, q_out=out)
    kept = slots >= 0
    want, size = turned(q, p, f, (24,), head_dim, False, 1.0)
    check(out[kept.to(DEV)], want[kept], size[kept], "q")
    assert (out.cpu()[~kept] == 9).all()
    want, size = turned(k, p, f, (24,), head_dim, False, 1.0)
    check(caches[0][slots[kept].to(DEV)], want[kept], size[kept], "k")
    assert torch.equal(caches[1].cpu()[slots[kept]], v[kept])
    free = torch.ones(9000, dtype=torch.bool)
    free[slots[kept]] = False
    assert (caches[0].cpu()[free] == 3).all() and (caches[1].cpu()[free] == 3).all()


def test_append_behind_32_bits_and_graph():
    # a cache of more than 2^32 bytes: slots at its end; the step captured once and replayed
    # with new tokens and lengths
    heads, head_dim, capacity, requests = 8, 128, 1200000, 2
    cache = torch.zeros(requests, capacity, heads * head_dim, dtype=BF16, device=DEV)
    v_cache = torch.zeros_like(cache)
    f, _ = ispa.rotary_frequencies(64)
    starts = torch.tensor([0, 2, 3], dtype=torch.int32, device=DEV)
    before = torch.tensor([capacity - 9, capacity - 5], dtype=torch.int32, device=DEV)
    q, k, v = (torch.randn(4, heads * head_dim, device=DEV).to(BF16) for _ in range(3))

    def step():
        slots, positions, lens = ispa.slot_map(starts, before, capacity, 4)
        return ispa.rotary_append(q, k, v, positions, slots, f, heads, cache, v_cache), lens

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lens = step()
    for turn in range(3):
        for t in (q, k, v):
            t.copy_(torch.randn(4, heads * head_dim, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        at = before.tolist()
        assert lens.tolist() == [at[0] + 2, at[1] + 1]
        p = torch.tensor([at[0], at[0] + 1, at[1]], dtype=torch.int32)
        want, size = turned(q[:3].cpu(), p[:, None], f.cpu(), (64,), head_dim, True, 1.0)
        check(out[:3], want, size, "q")
        want, size = turned(k[:3].cpu(), p[:, None], f.cpu(), (64,), head_dim, True, 1.0)
        rows = torch.stack((cache[0, at[0]], cache[0, at[0] + 1], cache[1, at[1]]))
        check(rows, want, size, "k")
        assert torch.equal(torch.stack((v_cache[0, at[0]], v_cache[0, at[0] + 1], v_cache[1, at[1]])), v[:3])
        before.copy_(lens)
