"""``LayerNorm`` as autograd sees it (no GPU needed): the kernels' place is taken by the formulas
in elementary operations, so that what is tested is the function around them."""

import pytest
import torch


def _forward(x, weight=None, bias=None, eps=1e-5, residual=None, stats=True):
    from paper_2608_15665_gb300 import firstorder as fo
    mean = x.mean(1)
    rstd = torch.rsqrt((x - mean[:, None]).square().mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return fo.LayerNormOut(y.detach(), mean.detach(), rstd.detach(), None)


def _backward(dy, x, weight, mean, rstd, dresidual=None, wdtype=None, want_weight=True,
              want_bias=True):
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy if weight is None else dy * weight
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return (dx.detach(), (dy * xh).sum(0).detach() if want_weight else None,
            dy.sum(0).detach() if want_bias else None)


@pytest.fixture
def fo(lib, monkeypatch):
    from paper_2608_15665_gb300 import firstorder
    monkeypatch.setattr(firstorder, "layer_norm", _forward)
    monkeypatch.setattr(firstorder, "layer_norm_backward", _backward)
    return firstorder


def _inputs(*needs):
    g = torch.Generator().manual_seed(4)
    made = [torch.randn(5, 12, generator=g, dtype=torch.float64),
            1.0 + torch.randn(12, generator=g, dtype=torch.float64),
            torch.randn(12, generator=g, dtype=torch.float64)]
    return [t.requires_grad_(n) for t, n in zip(made, needs or (True, True, True))]


def _want(ins, eps):
    ref = [t.detach().clone().requires_grad_(t.requires_grad) for t in ins]
    torch.nn.functional.layer_norm(ref[0], (12,), ref[1], ref[2], eps).square().sum().backward()
    return [t.grad for t in ref]


@pytest.mark.parametrize("extra,eps", [((), 1e-5), ((1e-5,), 1e-5), ((0.5,), 0.5)])
@pytest.mark.parametrize("needs", [(True, True, True), (True, False, True), (True, True, False),
                                   (True, False, False), (False, True, True)])
def test_gradients_with_and_without_an_eps(fo, extra, eps, needs):
    ins = _inputs(*needs)
    fo.LayerNorm.apply(*ins, *extra).square().sum().backward()
    for t, want in zip(ins, _want(ins, eps)):
        assert (t.grad is None) == (want is None)
        if want is not None:
            assert torch.allclose(t.grad, want, rtol=1e-9, atol=1e-12)


def test_a_second_derivative_is_refused(fo):
    """A penalty on the gradient is not silently taken for a constant."""
    x, w, b = _inputs()
    y = fo.LayerNorm.apply(x, w, b, 1e-5)
    dx, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (y.sum() + dx.square().sum()).backward()
