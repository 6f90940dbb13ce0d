"""Positions and frequencies of a call without rows are checked like those of any other."""

import pytest
import torch

import paper_2607_00712_amd as ispa

EMPTY = torch.zeros((0, 1), dtype=torch.int32)


@pytest.mark.parametrize("rows, positions", [(0, EMPTY), (0, EMPTY[:, 0]), (3, torch.zeros((3, 0), dtype=torch.int32))])
@pytest.mark.parametrize("freqs", [None, [1.0], 1.0])
def test_frequencies_that_are_no_tensor(rows, positions, freqs):
    with pytest.raises((TypeError, ValueError)):
        ispa._angles(positions, freqs, None, torch.device("cpu"), rows)


@pytest.mark.gpu
@pytest.mark.parametrize("turn", [lambda x, p, f: ispa.rotary(x, p, f, 2), lambda x, p, f: ispa.norm_rotary(x, x, p, f, 2),
                                  lambda x, p, f: ispa.norm_rotary_backward(x, x, x, x, p, f, 2)])
def test_calls_without_rows(turn):
    x, p, f = torch.zeros((0, 128), device="cuda"), EMPTY.to("cuda"), ispa.rotary_frequencies(32, device="cuda")[0]
    turn(x, p, f)
    turn(x, p[:, 0], f)
    for error, bad_p, bad_f in [(TypeError, p, None), (TypeError, None, f), (TypeError, p, f.float()), (ValueError, p, f[None]),
                                (ValueError, p.expand(0, 5).contiguous(), f), (TypeError, p.long(), f), (ValueError, p.cpu(), f)]:
        with pytest.raises(error):
            turn(x, bad_p, bad_f)
