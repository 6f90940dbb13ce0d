"""Tokens whose keys have no place in their cache: more new tokens than a ring's window,
tokens behind a cache's capacity. They attend like the others, so their queries are
turned; their keys and values are stored nowhere. Tolerances: those of the rotary and of
the shared attention tests.
"""

import pytest
import torch

import paper_2607_00712_amd as ispa
from test_gpu_attn_shared import check as check_attention, exact
from test_gpu_rotary import check, slots_of, turned

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32

# counts, before, capacity, sink, window, padding
BATCHES = [
    ([30, 2, 9], [0, 5, 40], 12, 4, 8, 3),       # a ring's window and more
    ([25, 0, 1], [7, 0, 100], 10, 0, 10, 0),     # without a sink
    ([9, 4, 30], [0, 20, 3], 16, 0, 0, 5),       # behind the capacity
    ([2100, 1], [3, 0], 40, 8, 32, 6),           # several tokens to a workgroup
]


def batch(case, heads, kv_heads, head_dim, dtype):
    counts, before, capacity, sink, window, pad = BATCHES[case]
    g = torch.Generator().manual_seed(case + heads)
    starts = [0]
    for m in counts:
        starts.append(starts[-1] + m)
    rows = starts[-1] + pad
    q = torch.randn(rows, heads * head_dim, generator=g).to(dtype)
    k, v = (torch.randn(rows, kv_heads * head_dim, generator=g).to(dtype) for _ in range(2))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    slots, positions, lens = ispa.slot_map(i32(starts), i32(before), capacity, rows, sink, window)
    want = slots_of(starts, before, capacity, rows, sink, window, 0)
    assert slots.tolist() == want[0] and any(s < 0 for s in want[0][:starts[-1]])
    return q, k, v, i32(starts), slots, positions, lens


@pytest.mark.parametrize("way", ["new", "given", "in place"])
@pytest.mark.parametrize("case", range(len(BATCHES)))
def test_queries_of_unplaced_tokens(case, way):
    heads, kv_heads, d = 4, 2, 64
    q, k, v, start, slots, positions, _ = batch(case, heads, kv_heads, d, BF16)
    counts, capacity = BATCHES[case][0], BATCHES[case][2]
    rows, real = len(q), sum(counts)
    f, _ = ispa.rotary_frequencies(d // 2, device="cpu")
    caches = [torch.full((len(counts), capacity, kv_heads * d), 3.0, dtype=BF16, device=DEV) for _ in range(2)]
    qg = q.to(DEV)
    out = {"new": None, "given": torch.full_like(qg, 9.0), "in place": qg}[way]
    got = ispa.rotary_append(qg, k.to(DEV), v.to(DEV), positions, slots, f.to(DEV), heads, *caches,
                             n_kv_heads=kv_heads, q_out=out, **({} if way == "new" else {"q_start": start}))
    torch.cuda.synchronize()
    p = positions.cpu()[:, None]
    want, size = turned(q, p, f, (d // 2,), d, True, 1.0)
    # (a new q_out has nothing to keep: its padding is turned too)
    n = rows if way == "new" else real
    check(got[:n], want[:n], size[:n], "q")
    if way == "given":
        assert (got[real:] == 9).all()
    if way == "in place":
        assert got is qg and torch.equal(got[real:].cpu(), q[real:])
    # keys and values: in their places alone
    slots, flat = slots.cpu(), [c.flatten(0, 1).cpu() for c in caches]
    kept = slots >= 0
    want, size = turned(k, p, f, (d // 2,), d, True, 1.0)
    check(flat[0][slots[kept]], want[kept], size[kept], "k")
    assert torch.equal(flat[1][slots[kept]], v[kept])
    free = torch.ones(len(flat[0]), dtype=torch.bool)
    free[slots[kept]] = False
    assert (flat[0][free] == 3).all() and (flat[1][free] == 3).all()


@pytest.mark.parametrize("case", range(3))
def test_attention_of_unplaced_tokens(case):
    # slot map, append, attention as a program runs them: every new token's output against
    # the prefix and what its cache holds, among them those that the cache does not keep
    heads, kv_heads, d, prefix = 4, 2, 64, 75
    q, k, v, start, slots, positions, lens = batch(case, heads, kv_heads, d, BF16)
    counts, capacity, real = BATCHES[case][0], BATCHES[case][2], sum(BATCHES[case][0])
    f, _ = ispa.rotary_frequencies(d // 2, device="cpu")
    g = torch.Generator().manual_seed(case)
    prefixes = [torch.randn(prefix, kv_heads * d, generator=g).to(BF16) for _ in range(2)]
    caches = [torch.randn(len(counts), capacity, kv_heads * d, generator=g).to(BF16).to(DEV) for _ in range(2)]
    turned_q = ispa.rotary_append(q.to(DEV), k.to(DEV), v.to(DEV), positions, slots, f.to(DEV), heads, *caches,
                                  n_kv_heads=kv_heads)
    out, lse = ispa.attn_shared(turned_q, *(p.to(DEV) for p in prefixes), *caches, start, lens, heads,
                                n_kv_heads=kv_heads, max_q=max(counts))
    torch.cuda.synchronize()
    # the queries from the definition, rounded as the call rounds them (at most one step of
    # bf16 apart, 2^-8, which moves a score by 2^-8 sum |q k|: below it is part of the bound)
    want_q, _ = turned(q, positions.cpu()[:, None], f, (d // 2,), d, True, 1.0)
    assert ((turned_q.cpu().double() - want_q).abs() <= want_q.abs() * 2.0 ** -8 + 2.0 ** -18).all()
    t = dict(q=turned_q.cpu(), k_prefix=prefixes[0], v_prefix=prefixes[1], k_cache=caches[0].cpu(),
             v_cache=caches[1].cpu(), q_start=start.cpu(), cache_lens=lens.cpu())
    want = exact(t, heads, kv_heads)
    check_attention(out[:real], lse[:, :real], tuple(w[:real] if i % 2 == 0 else w[:, :real] for i, w in enumerate(want)))


def test_given_rows_in_a_replayed_graph():
    # the count of real rows is read on the device: a captured step follows it
    heads, d, capacity, rows = 2, 64, 6, 20
    f, _ = ispa.rotary_frequencies(d // 2)
    q, k, v = (torch.randn(rows, heads * d, device=DEV).to(BF16) for _ in range(3))
    caches = [torch.zeros(1, capacity, heads * d, dtype=BF16, device=DEV) for _ in range(2)]
    start = torch.tensor([0, 11], dtype=torch.int32, device=DEV)
    before = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.empty(rows, heads * d, dtype=BF16, device=DEV)

    def step():
        slots, positions, _ = ispa.slot_map(start, before, capacity, rows, 0, capacity)
        return ispa.rotary_append(q, k, v, positions, slots, f, heads, *caches, q_out=out, q_start=start)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in (11, 0, 20, 7):
        start[1] = n
        before.fill_(n)
        out.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if n:
            p = (n + torch.arange(n, dtype=torch.int32))[:, None]
            want, size = turned(q[:n].cpu(), p, f.cpu(), (d // 2,), d, True, 1.0)
            check(out[:n], want, size, f"{n} rows")
        assert (out[n:] == 5).all()


def test_q_start_refusals():
    heads, d = 2, 64
    x = torch.zeros(3, heads * d, dtype=BF16, device=DEV)
    f, _ = ispa.rotary_frequencies(d // 2)
    p, s = torch.zeros(3, dtype=torch.int32, device=DEV), torch.arange(3, device=DEV)
    call = lambda start, **kw: ispa.rotary_append(x, x.clone(), x.clone(), p, s, f, heads, torch.zeros_like(x),
                                                  torch.zeros_like(x), q_start=start, **kw)
    good = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    call(good)
    for bad in (good.cpu(), good[:1], good[None]):
        with pytest.raises(ValueError):
            call(bad)
    with pytest.raises(TypeError):
        call(good.long())
