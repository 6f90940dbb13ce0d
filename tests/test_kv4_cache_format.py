"""A 4-bit cache is refused for another head_dim than it was made for, though its bytes would do:
a page of n tokens of 128 values is one of 2 n tokens of 64."""

import copy

import pytest
import torch

import paper_2607_00712_amd as ispa
from kv4_format import decode, encode

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


def test_how_far_a_number_is_off():
    """What include/ispa.h says of the rounding, over the whole range of fp32 (the GPU's numbers are
    the helper's: test_gpu_kv4.py)."""
    g = torch.Generator().manual_seed(0)
    for e in range(-149, 128):
        x = (1 + torch.rand(40, 32, generator=g, dtype=torch.float64)) * 2.0 ** e
        x[:, 1:] *= 2.0 ** -torch.randint(0, 6, (40, 31), generator=g) * (torch.randint(0, 2, (40, 31), generator=g) * 2 - 1)
        x = x.float().double()
        off, top = (decode(*encode(x)) - x).abs(), x.abs().amax(1, keepdim=True).expand(-1, 32)
        below, above = top < 1.25 * 2.0 ** -120, x.abs() > 7 * 2.0 ** 125
        assert (off <= torch.where(below, 2.0 ** -122, torch.where(above, x.abs() / 4, top / 5))).all()
        assert (decode(*encode(x))[above].abs() == 6 * 2.0 ** 125).all()
