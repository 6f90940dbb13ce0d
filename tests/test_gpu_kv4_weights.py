"""A bf16 output of the 4-bit attention has its softmax weights in 16 bits, however many rows meet
a key head and whatever the call was told of them: within the tolerance of single rows
(test_gpu_kv4.py: two bf16 parts leave 2^-16 of a weight)."""

import pytest
import torch

from test_gpu_kv4 import BF16, attend, check, exact, make, on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages", [4, 60])  # (an item to a workgroup, and equal runs with a join)
@pytest.mark.parametrize("rows", [9, 60, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_weights_of_many_rows(d, rows, pages):
    t = make([rows, 2], [32 * pages - 5, 70], 32, pages, 4, 2, d)
    g, want = on_gpu(t), exact(t, 4)
    for max_q in (1, rows, 5000):  # tiles of 16 rows, of 32, of 256
        print(f"attn_kv4 {rows} rows, head_dim {d}, {pages} pages, max_q {max_q}", flush=True)
        out, lse = attend(g, 4, max_q=max_q, out_dtype=BF16)
        torch.cuda.synchronize()
        check(out, lse, want, max_q, rows=1)
