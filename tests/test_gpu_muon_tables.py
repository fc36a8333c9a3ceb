"""The tables of a Muon context are in its workspace when zo_muon_create returns, whatever the
stream still had to do: the host memory that they come from is gone by then."""

import gc

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_they_are_there_when_the_handle_is(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    g = torch.Generator().manual_seed(2)
    Gs = [torch.randn(m, n, generator=g).to(gpu) for m, n in ((300, 260), (20, 20), (100, 700))]
    want = [o.clone() for o in fo.Orthogonalizer(Gs)()]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        with torch.cuda.stream(s):
            torch.cuda._sleep(100_000_000)
            op = fo.Orthogonalizer(Gs)
        assert s.query()                                 # nothing is left to be copied
        scribble = [torch.full((1 << 16,), 255, dtype=torch.uint8) for _ in range(64)]
        with torch.cuda.stream(s):
            got = [o.clone() for o in op()]
        s.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        op.close()
        del op, scribble
        gc.collect()
