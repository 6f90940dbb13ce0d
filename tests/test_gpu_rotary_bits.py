"""rotary's results to the bit: a caller that keeps turned keys across versions of the library gets
the same ones. The checksums are those of the kernel as it was first released; inputs are whole
numbers and powers of two, so that no generator stands behind them."""

import zlib

import pytest
import torch

import paper_2607_00712_amd as ispa

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
CRC = {  # interleaved, dtype, inverse
    (False, BF16, False): 1919418426, (False, BF16, True): 356828185,
    (False, F32, False): 591813647, (False, F32, True): 383249177,
    (True, BF16, False): 915410554, (True, BF16, True): 3838867521,
    (True, F32, False): 1281070427, (True, F32, True): 3400597267,
}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_keeps_its_bits(interleaved, dtype):
    rows, heads, d = 333, 3, 128
    i = torch.arange(rows * heads * d, dtype=torch.int64)
    x = (((i * 2654435761) % 65521 - 32760).double() / 4096).float().view(rows, heads * d).to(dtype).to(DEV)
    p = torch.stack([(i[:rows] * m) % 9973 for m in (7, 131, 1009)], 1).to(torch.int32).to(DEV)
    f = (torch.arange(1, 65, dtype=torch.float64) / 64).flip(0).to(DEV)  # (no power behind them either)
    for inverse in (False, True):
        out = ispa.rotary(x, p, f, heads, axes=(22, 21, 21), interleaved=interleaved, amplitude=1.25, inverse=inverse)
        crc = zlib.crc32(out.view(torch.uint8).cpu().numpy().tobytes())
        assert crc == CRC[interleaved, dtype, inverse]
