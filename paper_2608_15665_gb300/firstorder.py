"""Caller-side helpers around the first-order operators of the C ABI.

A model whose body is trained by subspace steps can train its tail by backpropagation,
which costs one backward pass through the tail alone and no activations of what lies
below it.  This module allocates the outputs and workspaces of those operators next to the
caller's tensors and launches them on PyTorch's current stream:

* ``layer_norm`` / ``layer_norm_backward`` -- the norm's forward and backward pass, and
  ``LayerNorm``, the two as one ``torch.autograd.Function``.

No arithmetic happens here.
"""

from typing import NamedTuple, Optional

import torch

from . import binding as zb


class LayerNormOut(NamedTuple):
    y: torch.Tensor
    mean: Optional[torch.Tensor]       # rows' statistics, fp32 (None: not asked for)
    rstd: Optional[torch.Tensor]
    h: Optional[torch.Tensor]          # x + residual, rounded to x's type (None: no residual)


def layer_norm(x, weight=None, bias=None, eps=1e-5, residual=None, stats=True):
    """LayerNorm over the last dimension of a rows x cols tensor, of x + residual where a
    residual is given (the sum comes back as ``h``)."""
    rows = x.shape[0]
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    h = torch.empty_like(y) if residual is not None else None
    mean = rstd = None
    if stats:
        mean = torch.empty(rows, dtype=torch.float32, device=x.device)
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    with torch.cuda.device(x.device):
        zb.zo_layernorm_forward(x, residual, weight, bias, eps, y, h, mean, rstd,
                                torch.cuda.current_stream())
    return LayerNormOut(y, mean, rstd, h)


def layer_norm_backward(dy, x, weight, mean, rstd, dresidual=None, wdtype=None, want_weight=True,
                        want_bias=True):
    """(dx, dweight, dbias) from the gradient of y and the forward pass's input (its ``h``
    where there was a residual) and statistics; dresidual is added to dx.  dweight and dbias
    have the weight's type (wdtype where there is none); None where not wanted."""
    if wdtype is None:
        wdtype = torch.float32 if weight is None else weight.dtype
    rows, cols = x.shape
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw = torch.empty(cols, dtype=wdtype, device=x.device) if want_weight else None
    db = torch.empty(cols, dtype=wdtype, device=x.device) if want_bias else None
    with torch.cuda.device(x.device):
        ws = None
        if want_weight or want_bias:
            ws = torch.empty(zb.zo_layernorm_workspace(rows, cols), dtype=torch.uint8,
                             device=x.device)
        zb.zo_layernorm_backward(dy, x, dresidual, weight, mean, rstd, dx, dw, db, ws,
                                 torch.cuda.current_stream())
    return dx, dw, db


class LayerNorm(torch.autograd.Function):
    """``LayerNorm.apply(x, weight, bias, eps)`` on a rows x cols tensor."""

    @staticmethod
    def forward(ctx, x, weight, bias, eps=1e-5):
        x = x.contiguous()
        out = layer_norm(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, out.mean, out.rstd)
        ctx.wdtype = (weight if weight is not None else bias).dtype \
            if weight is not None or bias is not None else None
        return out.y

    @staticmethod
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        _, need_w, need_b, _ = ctx.needs_input_grad
        dx, dw, db = layer_norm_backward(dy.contiguous(), x, weight, mean, rstd,
                                         wdtype=ctx.wdtype, want_weight=need_w, want_bias=need_b)
        return dx, dw, db, None
