"""Caller-side helpers around the first-order operators of the C ABI.

A model whose body is trained by subspace steps can train its tail by backpropagation,
which costs one backward pass through the tail alone and no activations of what lies
below it.  This module allocates the outputs and workspaces of those operators next to the
caller's tensors and launches them in the order of PyTorch's current stream:

* ``layer_norm`` / ``layer_norm_backward`` -- the norm's forward and backward pass, and
  ``LayerNorm``, the two as one ``torch.autograd.Function``; ``layer_norm_sync`` asks
  whether all of them went well;
* ``Orthogonalizer`` / ``Muon`` -- handles over matrices, bound to one stream.

No arithmetic happens here.
"""

from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as zb


class LayerNormOut(NamedTuple):
    y: torch.Tensor
    mean: Optional[torch.Tensor]       # rows' statistics, fp32 (None: not asked for)
    rstd: Optional[torch.Tensor]
    h: Optional[torch.Tensor]          # x + residual, rounded to x's type (None: no residual)


# The handle of a device's current stream, without a Stream object around it where PyTorch
# has that (about 1 us of a call that takes ten).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)
_empty, _empty_like = torch.empty, torch.empty_like
_contiguous = torch.contiguous_format
_F32 = torch.float32
_CODES = {torch.bfloat16: zb.ZO_BF16, torch.float32: zb.ZO_F32}


def _code(dtype, at, name):
    code = _CODES.get(dtype)
    return zb._code_of(dtype, at, name) if code is None else code     # (refuses)


def _call(fn, dev, at, *args):
    """A call of the C ABI on the current stream of device number `dev`."""
    if dev == torch.cuda.current_device():
        status = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _raw_stream(dev))
    if status:
        zb._check(status, at)


def _device_of(x, at):
    dev = x.get_device()
    if dev < 0:
        raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at, f"the tensors are on {x.device}, not on a GPU")
    return dev


def _refuse_grad(at, *tensors):
    """Outputs made through raw pointers have no history: where one would be recorded, an error."""
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at, "an input requires a gradient, which is not "
                             "recorded here: call LayerNorm.apply, or this under torch.no_grad()")


def layer_norm(x, weight=None, bias=None, eps=1e-5, residual=None, stats=True):
    """LayerNorm over the last dimension of a rows x cols tensor, of x + residual where a
    residual is given (the sum comes back as ``h``).  Its outputs have no history for autograd
    (``LayerNorm`` does that): inputs that require gradients are refused where they are recorded."""
    at = "layer_norm"
    _refuse_grad(at, x, weight, bias, residual)
    px, ldx = zb._rows(x, at, "x", None, None, None)
    shape, dt, device = x.shape, x.dtype, x.device
    rows, cols = shape
    dev = _device_of(x, at)
    pw = pb = pr = ph = pm = ps = h = mean = rstd = None
    wdt, ldr = _F32, 0
    if weight is not None:
        wdt = weight.dtype
        pw = zb._vector(weight, at, "weight", cols, wdt, device)
    elif bias is not None:
        wdt = bias.dtype
    if bias is not None:
        pb = zb._vector(bias, at, "bias", cols, wdt, device)
    # the outputs are contiguous: nothing of them needs a check
    y = _empty_like(x, memory_format=_contiguous)
    if residual is not None:
        pr, ldr = zb._rows(residual, at, "residual", shape, dt, device)
        h = _empty_like(y)
        ph = h.data_ptr()
    if stats:
        mean = _empty(rows, dtype=_F32, device=device)
        rstd = _empty_like(mean)
        pm, ps = mean.data_ptr(), rstd.data_ptr()
    _call(zb.LIB.zo_layernorm_forward, dev, at, px, ldx, pr, ldr, rows, cols, _code(dt, at, "x"),
          pw, pb, _code(wdt, at, "weight"), eps, y.data_ptr(), cols, ph, cols, pm, ps)
    return LayerNormOut(y, mean, rstd, h)


def layer_norm_backward(dy, x, weight, mean, rstd, dresidual=None, wdtype=None, want_weight=True,
                        want_bias=True):
    """(dx, dweight, dbias) from the gradient of y and the forward pass's input (its ``h``
    where there was a residual) and statistics; dresidual is added to dx.  dweight and dbias
    have the weight's type (wdtype where there is none); None where not wanted.  Like
    ``layer_norm``, without a history for autograd."""
    at = "layer_norm_backward"
    _refuse_grad(at, dy, x, weight, mean, rstd, dresidual)
    px, ldx = zb._rows(x, at, "x", None, None, None)
    shape, dt, device = x.shape, x.dtype, x.device
    rows, cols = shape
    dev = _device_of(x, at)
    pw = pdr = dw = db = pdw = pdb = pws = None
    lddr = ws_bytes = 0
    if weight is not None:
        wdtype = weight.dtype
        pw = zb._vector(weight, at, "weight", cols, wdtype, device)
    elif wdtype is None:
        wdtype = _F32
    pdy, lddy = zb._rows(dy, at, "dy", shape, dt, device)
    if dresidual is not None:
        pdr, lddr = zb._rows(dresidual, at, "dresidual", shape, dt, device)
    pm = zb._vector(mean, at, "mean", rows, _F32, device)
    ps = zb._vector(rstd, at, "rstd", rows, _F32, device)
    dx = _empty_like(x, memory_format=_contiguous)
    if want_weight:
        dw = _empty(cols, dtype=wdtype, device=device)
        pdw = dw.data_ptr()
    if want_bias:
        db = _empty(cols, dtype=wdtype, device=device) if dw is None else _empty_like(dw)
        pdb = db.data_ptr()
    if want_weight or want_bias:
        ws_bytes = zb.LIB.zo_layernorm_workspace(rows, cols)
        ws = _empty(ws_bytes, dtype=torch.uint8, device=device)
        pws = ws.data_ptr()
    _call(zb.LIB.zo_layernorm_backward, dev, at, pdy, lddy, px, ldx, pdr, lddr, rows, cols,
          _code(dt, at, "x"), pw, _code(wdtype, at, "weight"), pm, ps, dx.data_ptr(), cols, pdw,
          pdb, pws, ws_bytes)
    return dx, dw, db


def layer_norm_sync(device=None):
    """Waits for the current stream, and raises where a wait inside a layer norm's kernel has run
    out on this device since it was last asked (rows of that call are NaN then)."""
    with torch.cuda.device(device):
        zb.zo_layernorm_sync_status(torch.cuda.current_stream())


class LayerNorm(torch.autograd.Function):
    """``LayerNorm.apply(x, weight, bias, eps)`` on a rows x cols tensor.  Differentiable once:
    the gradients are the kernels', and asking for theirs is an error."""

    @staticmethod
    def forward(ctx, x, weight, bias, eps=1e-5):
        x = x.contiguous()
        out = layer_norm(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, out.mean, out.rstd)
        ctx.wdtype = (weight if weight is not None else bias).dtype \
            if weight is not None or bias is not None else None
        return out.y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        need_w, need_b = ctx.needs_input_grad[1:3]       # (there is no fourth without an eps)
        dx, dw, db = layer_norm_backward(dy.contiguous(), x, weight, mean, rstd,
                                         wdtype=ctx.wdtype, want_weight=need_w, want_bias=need_b)
        return dx, dw, db, None


ADJUST = {"none": zb.ZO_MUON_ADJUST_NONE, "aspect": zb.ZO_MUON_ADJUST_ASPECT,
          "rms": zb.ZO_MUON_ADJUST_RMS}


class _MuonContext:
    """A context over matrices and its workspace, on the stream that is PyTorch's current one
    when it is made (or `stream`).  A call under another current stream runs on the context's
    own all the same, after what that stream holds so far, and that stream goes on after it.
    (In a graph's capture too, where the context's own is not the legacy default stream, which
    CUDA keeps out of captures.)"""

    def __init__(self, weights, grads, momenta, stream, precise):
        self.ctx = None
        at = type(self).__name__
        if not weights:
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at, "need at least one matrix")
        dev = weights[0].device
        # (make_muon_matrix compares a matrix's own tensors)
        if any(W.device != dev for W in weights) or getattr(stream, "device", dev) != dev:
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at,
                             "the matrices and the stream have to be on one CUDA device")
        mats = [zb.make_muon_matrix(W, G, M) for W, G, M in zip(weights, grads, momenta)]
        if precise:
            for mat in mats:
                mat.grade = zb.ZO_MUON_GRADE_F32
        with torch.cuda.device(dev):
            current = torch.cuda.current_stream()
            self.stream = current if stream is None else stream
            if self.stream != current:      # what was filled for this context until now
                self.stream.wait_stream(current)
            with torch.cuda.stream(self.stream):
                self.workspace = torch.empty(zb.zo_muon_workspace(mats), dtype=torch.uint8,
                                             device=dev)
            self.ctx = zb.zo_muon_create(mats, self.workspace, self.stream)
        self.device = dev

    def _call(self, fn, *args):
        if _raw_stream(self.device.index) == self.stream.cuda_stream:
            fn(self.ctx, *args)
            return
        current = torch.cuda.current_stream(self.device)
        self.stream.wait_stream(current)
        fn(self.ctx, *args)
        current.wait_stream(self.stream)

    def sync(self):
        zb.zo_muon_sync_status(self.ctx)

    def close(self):
        if self.ctx is not None:
            zb.zo_muon_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Orthogonalizer(_MuonContext):
    """``op()`` orthogonalises every input by Newton-Schulz steps into its output (allocated
    with the input's shape and type if not given).  All on one CUDA device.  precise: products of
    fp32 grade for bf16 matrices of more than 128 rows (and columns) too."""

    def __init__(self, inputs, outputs=None, stream=None, precise=False):
        self.inputs = list(inputs)
        self.outputs = ([torch.empty(G.shape, dtype=G.dtype, device=G.device) for G in self.inputs]
                        if outputs is None else list(outputs))
        if len(self.outputs) != len(self.inputs):
            raise ValueError("as many outputs as inputs are needed")
        super().__init__(self.outputs, self.inputs, [None] * len(self.inputs), stream, precise)

    def __call__(self, steps=5, coeffs=None, eps=1e-7):
        self._call(zb.zo_orthogonalize, steps, coeffs, eps)
        return self.outputs


class Muon(_MuonContext):
    """The Muon optimiser over a list of weights (bf16 or fp32, on one CUDA device) whose
    gradients live in ``grads`` (allocated beside the weights, zero, if not given) and whose
    fp32 momenta in ``momenta``.  precise: as for ``Orthogonalizer``."""

    def __init__(self, weights, grads=None, momenta=None, stream=None, precise=False):
        self.weights = list(weights)
        self.grads = ([torch.zeros(W.shape, dtype=W.dtype, device=W.device) for W in self.weights]
                      if grads is None else list(grads))
        self.momenta = ([torch.zeros(W.shape, dtype=torch.float32, device=W.device)
                         for W in self.weights] if momenta is None else list(momenta))
        if not len(self.weights) == len(self.grads) == len(self.momenta):
            raise ValueError("as many gradients and momenta as weights are needed")
        super().__init__(self.weights, self.grads, self.momenta, stream, precise)

    def step(self, lr, momentum=0.95, nesterov=True, weight_decay=0.0, adjust="aspect", steps=5,
             coeffs=None, eps=1e-7):
        self._call(zb.zo_muon_step, momentum, nesterov, lr, weight_decay, ADJUST[adjust], steps,
                   coeffs, eps)
