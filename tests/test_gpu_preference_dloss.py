"""Gradients of the loss that are no numbers reach the rows that have a share in it, and no others: a
row whose derivative is 0 is not read and gets zeros."""

import pytest
import torch

from test_gpu_preference import TYPES, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [40, 3000, 20000])
@pytest.mark.parametrize("dloss", [float("inf"), float("-inf"), float("nan")])
def test_rows_without_a_share_get_zeros(lib, gpu, dloss, vocab, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    x, labels, offsets = make([3, 4], vocab, dtype, gpu, 5, tail=3, ignore=0.0)
    labels[1], labels[8] = -1, -7
    x[1] = float("nan")
    x[7:] = float("nan")                               # behind the last sequence
    got = fo.preference_loss(x, labels, offsets)
    d = fo.preference_loss_backward(x, labels, got.lse, got.dlogp, torch.tensor(dloss, device=gpu))
    mine = torch.tensor([True, False, True, True, True, True, True, False, False, False], device=gpu)
    assert (d[~mine] == 0).all()
    at = labels[mine][:, None]
    assert not torch.isfinite(d[mine].gather(1, at)).any()
    # a pair beyond the hinge has no share either
    ref = torch.tensor([-1e4, 1e4], device=gpu)
    got = fo.preference_loss(x, labels, offsets, ref, 0.1, "hinge")
    assert (got.dlogp == 0).all() and float(got.loss) == 0.0
    assert (fo.preference_loss_backward(x, labels, got.lse, got.dlogp, torch.tensor(dloss, device=gpu)) == 0).all()
