"""A 4-bit cache is refused for another head_dim than it was made for, though its bytes would do:
a page of n tokens of 128 values is one of 2 n tokens of 64."""

import copy

import pytest
import torch

import paper_2607_00712_amd as ispa

BF16 = torch.bfloat16
OTHER = {64: 128, 128: 64}


@pytest.mark.parametrize("page", [64, 256, 4096])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_of_another_head_dim(d, page):
    cache = ispa.kv4_cache(2, page, 3, d, device="cpu")
    assert cache.shape[2] % (OTHER[d] + OTHER[d] // 16) == 0  # (the bytes alone do not tell)
    for held, size in [(cache, None), (copy.deepcopy(cache), None), (cache.clone(), page), (cache, page)]:
        assert ispa._kv4_page_size(held, d, size) == page
        with pytest.raises(ValueError, match="pages of"):
            ispa._kv4_page_size(held, OTHER[d], size)
    with pytest.raises(ValueError, match="pages of"):
        ispa._kv4_page_size(cache, d, page // 2)
    assert ispa._kv4_page_size(cache.clone(), d, None) == page  # a tensor of the caller's own: its bytes


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_calls_for_another_head_dim(d):
    dev, page, kv, wrong = "cuda", 64, 2, OTHER[d]
    cache = ispa.kv4_cache(2, page, kv, d)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=dev)
    slots, at = torch.arange(3, device=dev), torch.arange(3, dtype=torch.int32, device=dev)
    start, lens = (torch.tensor(x, dtype=torch.int32, device=dev) for x in ([0, 3], [3]))
    row = lambda heads, width: torch.randn(3, heads * width, device=dev).to(BF16)
    f = {n: ispa.rotary_frequencies(n // 2, device=dev)[0] for n in (64, 128)}

    def calls(cache, width, **kw):
        x, q = row(kv, width), row(4, width)
        return [lambda: ispa.kv4_append(q, x, x, at, slots, f[width], 4, cache, table, n_kv_heads=kv, **kw),
                lambda: ispa.kv4_read(cache, table, slots, width, **kw),
                lambda: ispa.attn_kv4(q, cache, table, start, lens, 4, **kw)]

    for run in calls(cache, d) + calls(cache, d, page_size=page) + calls(cache.clone(), d, page_size=page):
        run()
    before = cache.clone()
    for run in calls(cache, wrong) + calls(before, wrong, page_size=page) + calls(cache, d, page_size=2 * page):
        with pytest.raises(ValueError, match="pages of"):
            run()
    torch.cuda.synchronize()
    assert torch.equal(cache, before)
    # the heads that a row is cut into decide its head_dim: half of them, and twice
    q = row(4, d)
    with pytest.raises(ValueError, match="pages of"):
        ispa.attn_kv4(q, cache, table, start, lens, 2 if d == 64 else 8)
