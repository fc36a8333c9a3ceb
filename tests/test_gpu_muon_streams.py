"""Muon handles stepped under other streams than their own, against the same work on one
stream, bit for bit.  Before each step the gradients are written on the current stream behind
50 ms of waiting, so that a step that did not wait for them would read the old ones."""

import pytest
import torch

pytestmark = pytest.mark.gpu

SHAPES = [(64, 64), (300, 520), (8, 900), (128, 100)]


def _data(dev, scale):
    g = torch.Generator().manual_seed(12)
    return [(torch.randn(m, n, generator=g) * scale).to(dev) for m, n in SHAPES]


def _train(dev, own, other):
    """Three steps of a handle on `own`, with everything else on `other`."""
    from paper_2608_15665_gb300 import firstorder as fo
    grads = _data(dev, 1.0)
    with torch.cuda.stream(other):
        other.wait_stream(torch.cuda.default_stream())
        W = [w.clone() for w in _data(dev, 0.1)]
        opt = fo.Muon(W, stream=own)
        out = []
        for t in range(3):
            torch.cuda._sleep(100_000_000)
            for k, g in enumerate(opt.grads):
                g.copy_(grads[k] * (0.5 ** t))
            opt.step(0.1, 0.9)
            out += [w.clone() for w in W]                    # reads what the step writes
        out += [m.clone() for m in opt.momenta]
    torch.cuda.synchronize()
    opt.sync()
    opt.close()
    return out


@pytest.mark.parametrize("own,other", [("side", "default"), ("default", "side"), ("side", "side2")])
def test_steps_are_ordered_with_the_current_stream(lib, gpu, own, other):
    streams = {"default": torch.cuda.default_stream(), "side": torch.cuda.Stream(),
               "side2": torch.cuda.Stream()}
    want = _train(gpu, torch.cuda.default_stream(), torch.cuda.default_stream())
    got = _train(gpu, streams[own], streams[other])
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_outputs_of_an_orthogonalizer_are_read_after_it(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    Gs = _data(gpu, 1.0)
    want = [o.clone() for o in fo.Orthogonalizer(Gs)()]
    work = [torch.zeros_like(G) for G in Gs]
    op = fo.Orthogonalizer(work)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(100_000_000)
        for w, G in zip(work, Gs):
            w.copy_(G)
        got = [o.clone() for o in op()]
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    op.close()


def test_a_step_captured_from_another_stream(lib, gpu):
    """A graph captured on one stream takes in the handle's own, which joins it and rejoins.
    (The legacy default stream can take no part in a capture: a handle's own has to be another.)"""
    from paper_2608_15665_gb300 import firstorder as fo
    grads = _data(gpu, 1.0)
    W = _data(gpu, 0.1)
    opt = fo.Muon(W, grads, stream=torch.cuda.Stream())
    opt.step(0.5, 0.9)                                       # set-up that a first launch does
    torch.cuda.synchronize()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        opt.step(0.5, 0.9)
    graph.replay()
    torch.cuda.synchronize()
    want = _data(gpu, 0.1)
    live = fo.Muon(want, grads)
    for _ in range(2):
        live.step(0.5, 0.9)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(W + opt.momenta, want + live.momenta))
