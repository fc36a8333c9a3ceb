"""Caller-side helpers around the first-order operators of the C ABI.

A model whose body is trained by subspace steps can train its tail by backpropagation,
which costs one backward pass through the tail alone and no activations of what lies
below it.  This module allocates the outputs and workspaces of those operators next to the
caller's tensors and launches them in the order of PyTorch's current stream:

* ``layer_norm`` / ``layer_norm_backward`` -- the norm's forward and backward pass, and
  ``LayerNorm``, the two as one ``torch.autograd.Function``; ``layer_norm_sync`` asks
  whether all of them went well;
* ``Orthogonalizer`` / ``Muon`` / ``AdamW`` -- handles over matrices (tensors of any shape for
  AdamW, whose states take 32 or 8 bits), bound to one stream;
* ``preference_loss`` / ``preference_loss_backward`` -- a loss over pairs of answers from their
  logits, and the logits' gradient; ``PreferenceLoss``, the two as one
  ``torch.autograd.Function``;
* ``gated_linear`` / ``gated_linear_backward`` -- the gated linear block of a feed-forward layer and
  its gradients, and ``GatedLinear``, the two as one ``torch.autograd.Function``;
  ``gated_linear_sync`` asks whether all of them went well.

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


def _refuse_grad(at, *tensors, function="LayerNorm"):
    """Outputs made through raw pointers have no history: where one would be recorded, an error."""
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at, "an input requires a gradient, which is not "
                             f"recorded here: call {function}.apply, or this under torch.no_grad()")


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


class _Handle:
    """A context of the library and its workspace, on the stream that is PyTorch's current one
    when it is made (or `stream`).  A call under another current stream runs on the context's
    own all the same, after what that stream holds so far, and that stream goes on after it.
    (In a graph's capture too, where the context's own is not the legacy default stream, which
    CUDA keeps out of captures.)"""

    ctx = None

    def _open(self, dev, stream, workspace_bytes, create):
        """Allocates workspace_bytes() and binds create(workspace, stream) on device `dev`."""
        with torch.cuda.device(dev):
            current = torch.cuda.current_stream()
            self.stream = current if stream is None else stream
            if self.stream != current:      # what was filled for this context until now
                self.stream.wait_stream(current)
            with torch.cuda.stream(self.stream):
                self.workspace = torch.empty(workspace_bytes(), dtype=torch.uint8, device=dev)
            self.ctx = create(self.workspace, self.stream)
        self.device = dev

    def _call(self, fn, *args):
        if _raw_stream(self.device.index) == self.stream.cuda_stream:
            fn(self.ctx, *args)
            return
        current = torch.cuda.current_stream(self.device)
        self.stream.wait_stream(current)
        fn(self.ctx, *args)
        current.wait_stream(self.stream)

    def _destroy(self, ctx):
        raise NotImplementedError

    def close(self):
        if self.ctx is not None:
            self._destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _MuonContext(_Handle):
    """A handle over matrices."""

    def __init__(self, weights, grads, momenta, stream, precise):
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
        self._open(dev, stream, lambda: zb.zo_muon_workspace(mats),
                   lambda workspace, on: zb.zo_muon_create(mats, workspace, on))

    def _destroy(self, ctx):
        zb.zo_muon_destroy(ctx)

    def sync(self):
        zb.zo_muon_sync_status(self.ctx)


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


class AdamWState(NamedTuple):
    """States of one tensor, an element each in the order of its rows: m and v in fp32, or m and
    sqrt(v) as float8_e4m3fn values of which each stands for itself times 2^(max(E, 40) - 134)
    with the exponent E of its 256 elements in m_exp and v_exp (uint8)."""
    m: torch.Tensor
    v: torch.Tensor
    m_exp: Optional[torch.Tensor] = None
    v_exp: Optional[torch.Tensor] = None


def adamw_state(weight, bits=32):
    """The states of a tensor before its first step: zero."""
    if bits not in (8, 32):
        raise zb.ZoError(zb.ZO_ERR_UNSUPPORTED, "adamw_state", "states are held in 8 or in 32 bits")
    n, dev = weight.numel(), weight.device
    if bits == 32:
        return AdamWState(torch.zeros(n, device=dev), torch.zeros(n, device=dev))
    m, v = (torch.zeros(n, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
            for _ in range(2))
    return AdamWState(m, v, *(torch.zeros(-(-n // zb.ADAMW_BLOCK), dtype=torch.uint8, device=dev)
                              for _ in range(2)))


class AdamW(_Handle):
    """The AdamW optimiser over a list of tensors (bf16 or fp32, on one CUDA device) whose
    gradients live in ``grads`` (allocated beside the weights, zero, if not given) and whose
    states, in 32 or 8 bits, in ``states``.  ``seed``: of the 8-bit states' random rounding (handles
    of the same seed take the same bits for their tensors of the same index: give each its own).  A
    handle is made once and kept: making it uploads its tables and waits for them.
    ``steps``: the number of steps taken, kept on the host; a step is told its number by it.
    ``count``: a one-element int64 tensor on the device, which takes its place: then a step that
    was captured into a graph may be replayed."""

    def __init__(self, weights, grads=None, states=None, bits=32, seed=0, count=None, stream=None):
        at = "AdamW"
        self.weights = list(weights)
        if not self.weights:
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at, "need at least one tensor")
        if bits not in (8, 32):
            raise zb.ZoError(zb.ZO_ERR_UNSUPPORTED, at, "states are held in 8 or in 32 bits")
        dev = self.weights[0].device
        if any(W.device != dev for W in self.weights) or getattr(stream, "device", dev) != dev:
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at,
                             "the tensors and the stream have to be on one CUDA device")
        if count is not None and (count.dtype != torch.int64 or count.numel() != 1
                                  or count.device != dev):
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at,
                             "count must be one int64 value beside the tensors")
        self.grads = ([torch.zeros(W.shape, dtype=W.dtype, device=W.device) for W in self.weights]
                      if grads is None else list(grads))
        self.states = ([adamw_state(W, bits) for W in self.weights] if states is None
                       else list(states))
        if not len(self.weights) == len(self.grads) == len(self.states):
            raise ValueError("as many gradients and states as weights are needed")
        if any((s.m_exp is None) != (bits == 32) for s in self.states):
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at, "states have exponents exactly with 8 bits")
        self.bits, self.count, self.steps = bits, count, 0
        tensors = [zb.make_adamw_tensor(W, G, *s)
                   for W, G, s in zip(self.weights, self.grads, self.states)]
        self._open(dev, stream, lambda: zb.zo_adamw_workspace(tensors, bits),
                   lambda workspace, on: zb.zo_adamw_create(tensors, bits, seed, workspace, on))

    def _destroy(self, ctx):
        zb.zo_adamw_destroy(ctx)

    def step(self, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, t=None):
        """One step.  t: its number, where it is not to be the one after the last."""
        if self.count is not None:
            if t is not None:
                raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, "AdamW.step",
                                 "the count on the device gives the step its number")
            self._call(zb.zo_adamw_step, 0, self.count, lr, betas[0], betas[1], eps, weight_decay)
            return
        if torch.cuda.is_current_stream_capturing():
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, "AdamW.step", "a captured step would take the "
                             "same number at every replay: give the handle a count on the device")
        t = self.steps + 1 if t is None else int(t)
        self._call(zb.zo_adamw_step, t, None, lr, betas[0], betas[1], eps, weight_decay)
        self.steps = t


class PreferenceOut(NamedTuple):
    loss: torch.Tensor                 # the pairs' mean, one fp32 value
    losses: torch.Tensor               # of every pair
    logps: torch.Tensor                # of every sequence, the chosen ones first
    lse: Optional[torch.Tensor]        # for the backward pass, per row (None: not asked for)
    dlogp: Optional[torch.Tensor]


PREFERENCES = {"sigmoid": zb.ZO_PREFERENCE_SIGMOID, "hinge": zb.ZO_PREFERENCE_HINGE,
               "square": zb.ZO_PREFERENCE_SQUARE}


def preference_loss(logits, labels, offsets, ref_logps=None, beta=0.1, kind="sigmoid",
                    smoothing=0.0, margin=0.0, average=False, grad=True, out=None):
    """The preference loss of pairs of answers from rows x vocab logits (bf16 or fp32) and the
    rows' labels (int64; below zero: the row does not count).  offsets (int64, 2 pairs + 1): the
    sequences' first rows, the chosen ones' and then the rejected ones', and the end.  ref_logps:
    the reference model's sums per sequence (fp32; none: zero).  average: means instead of sums.
    grad: also what the backward pass takes.  out: a one-element fp32 tensor for the loss, as a
    place in the losses of a subspace step.  Its outputs have no history for autograd
    (``PreferenceLoss`` does that)."""
    at = "preference_loss"
    _refuse_grad(at, logits, ref_logps, function="PreferenceLoss")
    if kind not in PREFERENCES:
        raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at, f"unknown kind {kind!r}")
    dev = _device_of(logits, at)
    px, ldl = zb._rows(logits, at, "logits", None, None, None)
    (rows, vocab), device = logits.shape, logits.device
    if offsets.dim() != 1 or offsets.shape[0] < 3 or offsets.shape[0] % 2 == 0:
        raise zb.ZoError(zb.ZO_ERR_SHAPE, at, "offsets must hold 2 pairs + 1 row numbers")
    pairs = offsets.shape[0] // 2
    plabels = zb._vector(labels, at, "labels", rows, torch.int64, device)
    poffsets = zb._vector(offsets, at, "offsets", 2 * pairs + 1, torch.int64, device)
    pref = zb._vector(ref_logps, at, "ref_logps", 2 * pairs, _F32, device)
    if out is None:
        loss = _empty((), dtype=_F32, device=device)
        ploss = loss.data_ptr()
    else:
        loss, ploss = out, zb._one_value(out, at, "out", device)
    losses = _empty(pairs, dtype=_F32, device=device)
    logps = _empty(2 * pairs, dtype=_F32, device=device)
    lse = dlogp = plse = pdlogp = None
    if grad:
        lse = _empty(rows, dtype=_F32, device=device)
        dlogp = _empty_like(lse)
        plse, pdlogp = lse.data_ptr(), dlogp.data_ptr()
    ws_bytes = zb.LIB.zo_preference_workspace(rows, vocab)
    ws = _empty(ws_bytes, dtype=torch.uint8, device=device)
    _call(zb.LIB.zo_preference_forward, dev, at, px, ldl, rows, vocab,
          _code(logits.dtype, at, "logits"), plabels, poffsets, pairs, pref, PREFERENCES[kind],
          beta, smoothing, margin, int(bool(average)), ploss, losses.data_ptr(), logps.data_ptr(),
          plse, pdlogp, ws.data_ptr(), ws_bytes)
    return PreferenceOut(loss, losses, logps, lse, dlogp)


def preference_loss_backward(logits, labels, lse, dlogp, dloss=None, out=None):
    """The logits' gradient from the forward pass's lse and dlogp (or any other loss's derivatives
    by the rows' log-probabilities) and the loss's own gradient (one fp32 value; none: 1).  out:
    where it goes, which may be the logits themselves.  Without a history for autograd."""
    at = "preference_loss_backward"
    _refuse_grad(at, logits, lse, dlogp, dloss, function="PreferenceLoss")
    dev = _device_of(logits, at)
    px, ldl = zb._rows(logits, at, "logits", None, None, None)
    (rows, vocab), device = logits.shape, logits.device
    plabels = zb._vector(labels, at, "labels", rows, torch.int64, device)
    plse = zb._vector(lse, at, "lse", rows, _F32, device)
    pdlogp = zb._vector(dlogp, at, "dlogp", rows, _F32, device)
    pdloss = zb._one_value(dloss, at, "dloss", device)
    if out is None:
        # rows as far apart as the logits', for accesses of the same alignment
        out = (_empty_like(logits, memory_format=_contiguous) if ldl == vocab else
               _empty((rows, ldl), dtype=logits.dtype, device=device)[:, :vocab])
    pd, ldd = zb._rows(out, at, "out", logits.shape, logits.dtype, device)
    _call(zb.LIB.zo_preference_backward, dev, at, px, ldl, rows, vocab,
          _code(logits.dtype, at, "logits"), plabels, plse, pdlogp, pdloss, pd, ldd)
    return out


class PreferenceLoss(torch.autograd.Function):
    """``PreferenceLoss.apply(logits, labels, offsets, ref_logps, beta, kind, smoothing, margin,
    average)``: the loss, differentiable once by the logits."""

    @staticmethod
    def forward(ctx, logits, labels, offsets, ref_logps=None, beta=0.1, kind="sigmoid",
                smoothing=0.0, margin=0.0, average=False):
        if ref_logps is not None and ref_logps.requires_grad:
            raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, "PreferenceLoss",
                             "the reference's log-probabilities get no gradient: detach them")
        out = preference_loss(logits, labels, offsets, ref_logps, beta, kind, smoothing, margin,
                              average, grad=ctx.needs_input_grad[0])
        ctx.save_for_backward(logits, labels, out.lse, out.dlogp)
        return out.loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        logits, labels, lse, dlogp = ctx.saved_tensors
        d = preference_loss_backward(logits, labels, lse, dlogp, dloss)
        return (d,) + (None,) * (len(ctx.needs_input_grad) - 1)


class GatedOut(NamedTuple):
    h: torch.Tensor
    gate: Optional[torch.Tensor]       # X Wg^T and X Wu^T for the backward pass (None: not kept)
    up: Optional[torch.Tensor]


ACTIVATIONS = {"silu": zb.ZO_GATED_SILU, "gelu": zb.ZO_GATED_GELU_TANH}
_BF16 = torch.bfloat16


def _activation(act, at):
    if act not in ACTIVATIONS:
        raise zb.ZoError(zb.ZO_ERR_INVALID_ARG, at, f"unknown activation {act!r}")
    return ACTIVATIONS[act]


def _gated_inputs(x, w_gate, w_up, at):
    dev = _device_of(x, at)
    px = zb._rows(x, at, "x", None, _BF16, None)
    pg = zb._rows(w_gate, at, "w_gate", None, _BF16, x.device)
    if w_gate.shape[1] != x.shape[1]:
        raise zb.ZoError(zb.ZO_ERR_SHAPE, at, f"w_gate has shape {tuple(w_gate.shape)}, expected "
                                              f"(F, {x.shape[1]})")
    return dev, px, pg, zb._rows(w_up, at, "w_up", w_gate.shape, _BF16, x.device)


def gated_linear(x, w_gate, w_up, act="silu", save=False):
    """h = act(x w_gate^T) (x w_up^T) of a tokens x D matrix and F x D weights (bf16; D and F
    multiples of 8), with act "silu" or "gelu" (by tanh).  save: both products too, for the
    backward pass.  Its outputs have no history for autograd (``GatedLinear`` does that)."""
    at = "gated_linear"
    _refuse_grad(at, x, w_gate, w_up, function="GatedLinear")
    code = _activation(act, at)
    dev, px, pg, pu = _gated_inputs(x, w_gate, w_up, at)
    (T, D), F = x.shape, w_gate.shape[0]
    h = _empty((T, F), dtype=_BF16, device=x.device)
    gate = up = pgate = pup = None
    if save:
        gate, up = _empty_like(h), _empty_like(h)
        pgate, pup = gate.data_ptr(), up.data_ptr()
    _call(zb.LIB.zo_gated_forward, dev, at, *px, T, D, *pg, *pu, F, code, h.data_ptr(), F, pgate, F,
          pup, F)
    return GatedOut(h, gate, up)


def gated_linear_backward(dh, x, w_gate, w_up, gate, up, act="silu", want_x=True, want_weights=True):
    """(dx, dw_gate, dw_up) from the gradient of h and the forward pass's inputs and products; None
    where not wanted.  Like ``gated_linear``, without a history for autograd."""
    at = "gated_linear_backward"
    _refuse_grad(at, dh, x, w_gate, w_up, gate, up, function="GatedLinear")
    code = _activation(act, at)
    dev, px, pg, pu = _gated_inputs(x, w_gate, w_up, at)
    (T, D), F, device = x.shape, w_gate.shape[0], x.device
    ins = [zb._rows(t, at, name, (T, F), _BF16, device)
           for name, t in (("dh", dh), ("gate", gate), ("up", up))]
    dx = dwg = dwu = pdx = pdwg = pdwu = None
    if want_x:
        dx = _empty((T, D), dtype=_BF16, device=device)
        pdx = dx.data_ptr()
    if want_weights:
        dwg, dwu = (_empty((F, D), dtype=_BF16, device=device) for _ in range(2))
        pdwg, pdwu = dwg.data_ptr(), dwu.data_ptr()
    ws_bytes = zb.LIB.zo_gated_workspace(T, D, F)
    ws = _empty(ws_bytes, dtype=torch.uint8, device=device)
    _call(zb.LIB.zo_gated_backward, dev, at, *ins[0], *px, T, D, *pg, *pu, F, code, *ins[1], *ins[2],
          pdx, D, pdwg, D, pdwu, D, ws.data_ptr(), ws_bytes)
    return dx, dwg, dwu


def gated_linear_sync(device=None):
    """Waits for the current stream, and raises where a wait inside a gated linear block's kernel has
    run out on this device since it was last asked (results of that call are NaN then, in part or whole)."""
    with torch.cuda.device(device):
        zb.zo_gated_sync_status(torch.cuda.current_stream())


def _packed(t):
    """A matrix as the kernels take it: rows without gaps, on a 16-byte boundary."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class GatedLinear(torch.autograd.Function):
    """``GatedLinear.apply(x, w_gate, w_up, act)`` on a tokens x D matrix.  Differentiable once."""

    @staticmethod
    def forward(ctx, x, w_gate, w_up, act="silu"):
        x = _packed(x)
        out = gated_linear(x, w_gate, w_up, act, save=any(ctx.needs_input_grad[:3]))
        ctx.save_for_backward(x, w_gate, w_up, out.gate, out.up)
        ctx.act = act
        return out.h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        x, w_gate, w_up, gate, up = ctx.saved_tensors
        need_x, need_g, need_u = ctx.needs_input_grad[:3]
        dx, dwg, dwu = gated_linear_backward(_packed(dh), x, w_gate, w_up, gate, up, ctx.act,
                                             want_x=need_x, want_weights=need_g or need_u)
        return dx, dwg if need_g else None, dwu if need_u else None, None
