"""The 4-bit cache's format in 64 bits, for the tests: 32 values of a head as 4-bit numbers
of one power of two (layout: include/ispa.h)."""

import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
NUMBERS = torch.cat((GRID, -GRID))


def encode(x):
    """x [..., d] fp64 as codes [..., d] and powers (plus 127) [..., d / 32]."""
    x = x.double().unflatten(-1, (-1, 32))
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[..., None], torch.zeros_like(x), x)
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)  # top = m 2^e, 0.5 <= m < 1, and 7 = 0.875 2^3
    e = torch.where(m > 0.875, e - 2, e - 3).clamp(-120, 125)
    e = torch.where(top == 0, torch.full_like(e, -120), e)
    y = x / torch.exp2(e.double())[..., None]
    off = (y.abs()[..., None] - GRID).abs()
    best = off.amin(-1, keepdim=True)
    near = off == best  # one number, or the two beside a border: the even code
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(near.sum(-1) > 1, even.int().argmax(-1), near.int().argmax(-1))
    code = code + 8 * (y < 0)
    return code.flatten(-2).to(torch.uint8), torch.where(bad, torch.full_like(e, 128), e).add(127).to(torch.uint8)


def decode(code, power):
    """Values fp64 [..., d] of codes [..., d] and powers [..., d / 32]."""
    x = NUMBERS[code.long()].unflatten(-1, (-1, 32)) * torch.exp2(power.double() - 127)[..., None]
    return torch.where((power == 255)[..., None], torch.full_like(x, float("nan")), x).flatten(-2)


def pack(k, v):
    """Pages [n, heads, bytes] of keys and values, each (codes, powers) with [n, heads, page, ...]."""
    halves = [(c[..., 0::2] | c[..., 1::2] << 4).flatten(2) for c, _ in (k, v)]
    return torch.cat((*halves, torch.stack((k[1], v[1]), dim=3).flatten(2)), dim=2).contiguous()


def unpack(cache, d):
    """((codes, powers) of the keys, of the values), [n, heads, page, ...] each."""
    n, heads, nbytes = cache.shape
    page = nbytes // (d + d // 16)
    powers = cache[:, :, page * d:].view(n, heads, page, 2, d // 32)
    out = []
    for i in range(2):
        b = cache[:, :, i * page * d // 2:(i + 1) * page * d // 2].reshape(n, heads, page, d // 2)
        out.append((torch.stack((b & 15, b >> 4), -1).flatten(-2), powers[:, :, :, i]))
    return out
