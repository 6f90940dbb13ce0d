"""kv4_read refuses what one launch does not hold: 256 threads to a workgroup, 8 values of k or v to a
thread, fewer than 2^32 threads in all. (Pointers here are fake and never read.)"""

import pytest

import paper_2607_00712_amd as ispa
from test_kv4_abi import READ
from test_operators_abi import call


@pytest.mark.parametrize("heads, head_dim, rows", [(1, 64, (1 << 28) - 1), (1, 64, (1 << 28) - 15), (1, 128, (1 << 27) - 1),
                                                   (3, 64, ((1 << 34) - 1023) // 192 + 1), (16, 64, 1 << 24)])
def test_rows_of_one_launch(heads, head_dim, rows):
    assert (rows * heads * head_dim // 4 + 255) // 256 * 256 >= 1 << 32  # threads
    far = dict(slots=1 << 44, k=1 << 45, v=1 << 46)
    assert call("ispa_kv4_read", READ, n_kv_heads=heads, head_dim=head_dim, rows=rows, **far) == ispa.ISPA_ERR_INVALID_ARG
