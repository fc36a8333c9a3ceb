"""How the Muon handles order their stream against PyTorch's current one (no GPU needed): with
fake streams, and the library's calls recorded in place of being made."""

import contextlib

import pytest
import torch


class FakeStream:
    def __init__(self, name, log):
        self.name, self.log, self.cuda_stream = name, log, id(self)

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))


class Cuda:
    """The current stream, and what was called in what order."""

    def __init__(self):
        self.log = []
        self.current = self.stream("default")

    def stream(self, name):
        return FakeStream(name, self.log)

    @contextlib.contextmanager
    def use(self, stream):
        before, self.current = self.current, stream
        yield
        self.current = before


@pytest.fixture
def cuda(lib, monkeypatch):
    from paper_2608_15665_gb300 import firstorder as fo
    c = Cuda()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: c.current)
    monkeypatch.setattr(torch.cuda, "device", lambda dev: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", c.use)
    monkeypatch.setattr(fo, "_raw_stream", lambda dev: c.current.cuda_stream)
    monkeypatch.setattr(lib, "make_muon_matrix", lambda W, G, M: object())
    monkeypatch.setattr(lib, "zo_muon_workspace", lambda mats: 256)
    for name in ("zo_muon_create", "zo_muon_destroy", "zo_orthogonalize", "zo_muon_step"):
        monkeypatch.setattr(lib, name, lambda *a, name=name: c.log.append(name))
    return c


def _handles(fo, stream):
    W = [torch.ones(4, 8)]
    return [lambda: fo.Muon(W, stream=stream), lambda: fo.Orthogonalizer(W, stream=stream)]


@pytest.mark.parametrize("which", [0, 1])
def test_a_stream_of_its_own_waits_for_what_was_filled_before(cuda, which):
    from paper_2608_15665_gb300 import firstorder as fo
    s = cuda.stream("s")
    op = _handles(fo, s)[which]()
    assert op.stream is s
    assert cuda.log == [("s", "waits for", "default"), "zo_muon_create"]
    op.close()


@pytest.mark.parametrize("which", [0, 1])
def test_the_current_stream_waits_for_nothing(cuda, which):
    from paper_2608_15665_gb300 import firstorder as fo
    op = _handles(fo, None)[which]()
    assert op.stream is cuda.current
    assert cuda.log == ["zo_muon_create"]
    op.close()


def _call(op):
    op.step(0.1) if hasattr(op, "step") else op()


@pytest.mark.parametrize("which", [0, 1])
def test_a_call_under_another_stream_lies_between_its_work(cuda, which):
    from paper_2608_15665_gb300 import firstorder as fo
    op, s = _handles(fo, None)[which](), cuda.stream("s")
    del cuda.log[:]
    name = ("zo_muon_step", "zo_orthogonalize")[which]
    with torch.cuda.stream(s):
        _call(op)
    assert cuda.log == [("default", "waits for", "s"), name, ("s", "waits for", "default")]
    del cuda.log[:]
    _call(op)                                                # and under its own
    assert cuda.log == [name]
