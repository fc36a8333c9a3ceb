"""``layer_norm`` and ``layer_norm_backward`` refuse inputs whose gradients would be lost (no GPU
needed: what is not refused for that goes on to be refused for lying on the CPU)."""

import pytest
import torch


def _refusal(lib, call):
    with pytest.raises(lib.ZoError) as e:
        call()
    assert e.value.status == lib.ZO_ERR_INVALID_ARG
    return "requires a gradient" in str(e.value)


FORWARD = ("x", "weight", "bias", "residual")
BACKWARD = ("dy", "x", "weight", "mean", "rstd", "dresidual")


def _tensors(names):
    size = {"weight": (6,), "bias": (6,), "mean": (4,), "rstd": (4,)}
    return {n: torch.ones(size.get(n, (4, 6))) for n in names}


@pytest.mark.parametrize("which", FORWARD)
def test_forward(lib, which):
    from paper_2608_15665_gb300 import firstorder as fo
    kw = _tensors(FORWARD)
    assert not _refusal(lib, lambda: fo.layer_norm(**kw))
    kw[which].requires_grad_()
    assert _refusal(lib, lambda: fo.layer_norm(**kw))
    with torch.no_grad():
        assert not _refusal(lib, lambda: fo.layer_norm(**kw))
    assert not _refusal(lib, lambda: fo.LayerNorm.apply(kw["x"], kw["weight"], kw["bias"]))


@pytest.mark.parametrize("which", BACKWARD)
def test_backward(lib, which):
    from paper_2608_15665_gb300 import firstorder as fo
    kw = _tensors(BACKWARD)
    assert not _refusal(lib, lambda: fo.layer_norm_backward(**kw))
    kw[which].requires_grad_()
    assert _refusal(lib, lambda: fo.layer_norm_backward(**kw))
    with torch.no_grad():
        assert not _refusal(lib, lambda: fo.layer_norm_backward(**kw))
