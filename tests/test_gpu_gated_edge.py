"""The gated block's gradients where dG is beyond bf16's largest number and still fp32's: it rounds to
infinity, in sums of two bf16 as in one, and its rows of dX are infinite and no NaN."""

import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.mark.parametrize("T", [5, 128, 200])
def test_gradients_that_round_to_infinity(lib, gpu, T):
    from paper_2608_15665_gb300 import firstorder as fo
    D, F = 64, 72
    x, wg, wu = (torch.ones(n, D, dtype=BF, device=gpu) for n in (T, F, F))
    wu.zero_()
    dh = torch.zeros(T, F, dtype=BF, device=gpu)
    dh[1, 3], dh[2, 3] = 2.0 ** 100, -2.0 ** 100
    # silu'(8) = 1.0023: dG = 2^127 x 1.9969 lies between 2^128 less half a step of bf16's and 2^128
    # (and dU = 2^103)
    gate, up = torch.full_like(dh, 8.0), torch.full_like(dh, 1.9921875 * 2.0 ** 27)
    dx, dwg, _ = fo.gated_linear_backward(dh, x, wg, wu, gate, up)
    inf = float("inf")
    assert (dx[1] == inf).all() and (dx[2] == -inf).all()
    assert (dx[0] == 0).all() and (dx[3:] == 0).all()
    # (infinities of both signs meet in dWg's row 3)
    assert torch.isnan(dwg[3]).all() and (dwg[:3] == 0).all() and (dwg[4:] == 0).all()
