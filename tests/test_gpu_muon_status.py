"""What a Muon context reports when a wait on the device has run out: ZO_ERR_TIMEOUT once, and
then the results of a context that never had one.  No wait runs out here: the test sets the
status word, the first of the caller's workspace, as a kernel that gave up does."""

import pytest
import torch

pytestmark = pytest.mark.gpu

SHAPES = [(300, 260), (48, 7680), (100, 96), (8, 700)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_wait_that_ran_out_is_reported_once(lib, gpu, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    g = torch.Generator().manual_seed(3)
    Gs = [torch.randn(m, n, generator=g).to(dtype).to(gpu) for m, n in SHAPES]
    want = [o.clone() for o in fo.Orthogonalizer(Gs)()]
    op = fo.Orthogonalizer(Gs)
    op()
    op.sync()
    op.workspace[:4].view(torch.int32).fill_(1)
    with pytest.raises(lib.ZoError) as e:
        op.sync()
    assert e.value.status == lib.ZO_ERR_TIMEOUT
    op.sync()                                    # cleared
    for o in op.outputs:
        o.fill_(float("nan"))
    op()
    op.sync()
    for a, b in zip(op.outputs, want):
        assert torch.equal(a, b)
    op.close()
