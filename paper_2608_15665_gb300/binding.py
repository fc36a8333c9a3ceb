"""ctypes binding of the C ABI in include/zo.h (argument marshalling only).

Every function here has the name of the C entry point it calls and does nothing
but convert arguments (torch tensors -> device pointers, Python scalars -> C
types) and turn a non-zero status into ``ZoError``.  All computation runs in
the CUDA library ``libsubzero_zo.so``; if that library is missing, importing
this module fails -- there is no fallback.
"""

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsubzero_zo.so")

ZO_OK = 0
ZO_ERR_INVALID_ARG = 1
ZO_ERR_SHAPE = 2
ZO_ERR_ALIGN = 3
ZO_ERR_DTYPE = 4
ZO_ERR_CUDA = 5
ZO_ERR_TIMEOUT = 6
ZO_ERR_UNSUPPORTED = 7
ZO_ERR_NOMEM = 8

ZO_F32 = 0
ZO_BF16 = 1

ZO_SCHEME_CENTRAL = 0
ZO_SCHEME_FORWARD = 1
ZO_SCHEME_DIRECT = 2

ZO_OPT_ADAM = 0
ZO_OPT_SGD = 1
ZO_OPT_MUON = 2

ZO_MUON_ADJUST_NONE = 0
ZO_MUON_ADJUST_ASPECT = 1
ZO_MUON_ADJUST_RMS = 2
ZO_MUON_GRADE_DTYPE = 0
ZO_MUON_GRADE_F32 = 1

ZO_OPTION_WPASS_PATH = 0
ZO_OPTION_TIMING = 1
ZO_OPTION_TEST_WAIT_TIMEOUT = 2
ZO_OPTION_LINEAR_TILE = 3
ZO_OPTION_PAIR_MMA = 4


class ZoError(RuntimeError):
    def __init__(self, status, where, detail=""):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status}) {detail}".rstrip())


class zo_matrix(ctypes.Structure):
    _fields_ = [
        ("W", ctypes.c_void_p),
        ("m", ctypes.c_int64),
        ("n", ctypes.c_int64),
        ("ldw", ctypes.c_int64),
        ("dtype", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("U", ctypes.c_void_p),
        ("V", ctypes.c_void_p),
        ("M", ctypes.c_void_p),
        ("Vm", ctypes.c_void_p),
    ]


class zo_muon_matrix(ctypes.Structure):
    _fields_ = [
        ("W", ctypes.c_void_p),
        ("G", ctypes.c_void_p),
        ("M", ctypes.c_void_p),
        ("m", ctypes.c_int64),
        ("n", ctypes.c_int64),
        ("ldw", ctypes.c_int64),
        ("ldg", ctypes.c_int64),
        ("dtype", ctypes.c_int32),
        ("grad_dtype", ctypes.c_int32),
        ("grade", ctypes.c_int32),
    ]


_c = ctypes
_SIGNATURES = {
    "zo_create": (_c.c_int32, [_c.POINTER(_c.c_void_p), _c.POINTER(zo_matrix), _c.c_int32,
                               _c.c_int32, _c.c_int32, _c.c_uint64, _c.c_uint32, _c.c_void_p]),
    "zo_destroy": (_c.c_int32, [_c.c_void_p]),
    "zo_refresh": (_c.c_int32, [_c.c_void_p, _c.c_uint32, _c.c_int32]),
    "zo_init_subspace": (_c.c_int32, [_c.c_void_p, _c.c_uint32]),
    "zo_perturb": (_c.c_int32, [_c.c_void_p, _c.c_uint32, _c.c_int32, _c.c_float, _c.c_int32,
                                _c.c_float, _c.c_float]),
    "zo_step": (_c.c_int32, [_c.c_void_p, _c.c_uint32, _c.c_int32, _c.c_void_p, _c.c_int32,
                             _c.c_int32, _c.c_int32, _c.c_int32, _c.c_float, _c.c_float,
                             _c.c_float, _c.c_float, _c.c_float, _c.c_int32, _c.c_float,
                             _c.c_void_p]),
    "zo_mezo_perturb": (_c.c_int32, [_c.c_void_p, _c.c_uint32, _c.c_float]),
    "zo_linear_prepare": (_c.c_int32, [_c.c_void_p, _c.c_uint32, _c.c_int32, _c.c_float,
                                       _c.c_int32, _c.c_float, _c.c_float]),
    "zo_linear_perturbed": (_c.c_int32, [_c.c_void_p, _c.c_int32, _c.c_void_p, _c.c_int64,
                                         _c.c_int64, _c.c_void_p, _c.c_int64]),
    "zo_sync_status": (_c.c_int32, [_c.c_void_p]),
    "zo_set_option": (_c.c_int32, [_c.c_void_p, _c.c_int32, _c.c_int64]),
    "zo_get_timing": (_c.c_int32, [_c.c_void_p, _c.POINTER(_c.c_double), _c.POINTER(_c.c_int64)]),
    "zo_wpass_path": (_c.c_int32, [_c.c_void_p]),
    "zo_linear_tiling": (_c.c_int32, [_c.c_void_p]),
    "zo_kernel_launches": (_c.c_int64, [_c.c_void_p]),
    "zo_philox_fill": (_c.c_int32, [_c.c_uint64, _c.c_uint32, _c.c_uint32, _c.c_uint32,
                                    _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "zo_normal_fill": (_c.c_int32, [_c.c_uint64, _c.c_uint32, _c.c_uint32, _c.c_uint32,
                                    _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "zo_perturb_noalloc": (_c.c_int32, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64,
                                        _c.c_int32, _c.c_void_p, _c.c_void_p, _c.c_int32,
                                        _c.c_uint64, _c.c_uint32, _c.c_uint32, _c.c_int32,
                                        _c.c_float, _c.c_int32, _c.c_float, _c.c_float,
                                        _c.c_void_p]),
    "zo_layernorm_forward": (_c.c_int32, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64,
                                          _c.c_int64, _c.c_int64, _c.c_int32, _c.c_void_p,
                                          _c.c_void_p, _c.c_int32, _c.c_float, _c.c_void_p,
                                          _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_void_p,
                                          _c.c_void_p, _c.c_void_p]),
    "zo_layernorm_workspace": (_c.c_int64, [_c.c_int64, _c.c_int64]),
    "zo_layernorm_backward": (_c.c_int32, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64,
                                           _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64,
                                           _c.c_int32, _c.c_void_p, _c.c_int32, _c.c_void_p,
                                           _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p,
                                           _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "zo_layernorm_sync_status": (_c.c_int32, [_c.c_void_p]),
    "zo_muon_workspace": (_c.c_int64, [_c.c_void_p, _c.c_int32]),
    "zo_muon_create": (_c.c_int32, [_c.POINTER(_c.c_void_p), _c.c_void_p, _c.c_int32, _c.c_void_p,
                                    _c.c_int64, _c.c_void_p]),
    "zo_muon_destroy": (_c.c_int32, [_c.c_void_p]),
    "zo_orthogonalize": (_c.c_int32, [_c.c_void_p, _c.c_int32, _c.c_void_p, _c.c_float]),
    "zo_muon_step": (_c.c_int32, [_c.c_void_p, _c.c_float, _c.c_int32, _c.c_float, _c.c_float,
                                  _c.c_int32, _c.c_int32, _c.c_void_p, _c.c_float]),
    "zo_muon_sync_status": (_c.c_int32, [_c.c_void_p]),
    "zo_muon_launches": (_c.c_int64, [_c.c_void_p]),
    "zo_status_string": (_c.c_char_p, [_c.c_int32]),
    "zo_last_error": (_c.c_char_p, []),
}


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with paper_2608_15665_gb300.build.build() "
            "(nvcc, sm_103a). There is no CPU fallback.")
    lib = ctypes.CDLL(LIB_PATH)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


LIB = _load()


def status_string(status):
    return LIB.zo_status_string(int(status)).decode()


def zo_last_error():
    return LIB.zo_last_error().decode()


def _check(status, where):
    if status != ZO_OK:
        raise ZoError(status, where, zo_last_error())


def _ptr(t):
    """Device pointer of a tensor (or an int address, or None -> NULL)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream_handle(stream):
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_matrix(W, U, V, M, Vm):
    """zo_matrix for torch tensors: W (m x n, bf16/fp32, row stride ldw), U (m x r),
    V (n x r), M and Vm (r x r), all fp32 except W."""
    import torch
    if W.dtype == torch.bfloat16:
        dt = ZO_BF16
    elif W.dtype == torch.float32:
        dt = ZO_F32
    else:
        raise ZoError(ZO_ERR_DTYPE, "make_matrix", str(W.dtype))
    if W.dim() != 2 or W.stride(1) != 1:
        raise ZoError(ZO_ERR_SHAPE, "make_matrix", "W must be 2-D with unit column stride")
    for name, t in (("U", U), ("V", V), ("M", M), ("Vm", Vm)):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ZoError(ZO_ERR_DTYPE, "make_matrix", f"{name} must be contiguous fp32")
    return zo_matrix(_ptr(W), W.shape[0], W.shape[1], W.stride(0), dt, 0, _ptr(U), _ptr(V),
                     _ptr(M), _ptr(Vm))


def zo_create(mats, r, q, seed, matrix_index_base=0, stream=None):
    arr = (zo_matrix * len(mats))(*mats)
    ctx = ctypes.c_void_p()
    _check(LIB.zo_create(ctypes.byref(ctx), arr, len(mats), int(r), int(q), int(seed) & (2**64 - 1),
                         int(matrix_index_base), _stream_handle(stream)), "zo_create")
    return ctx


def zo_destroy(ctx):
    _check(LIB.zo_destroy(ctx), "zo_destroy")


def zo_refresh(ctx, refresh_idx, reset_moments=False):
    _check(LIB.zo_refresh(ctx, int(refresh_idx), int(bool(reset_moments))), "zo_refresh")


def zo_init_subspace(ctx, refresh_idx=0):
    _check(LIB.zo_init_subspace(ctx, int(refresh_idx)), "zo_init_subspace")


def zo_perturb(ctx, t, qa, ca, qb, cb, eps):
    _check(LIB.zo_perturb(ctx, int(t), int(qa), float(ca), int(qb), float(cb), float(eps)),
           "zo_perturb")


def zo_step(ctx, t, adam_t, losses, scheme, eps, lr, beta1, beta2, eps_adam, restore_query,
            restore_coef, optimizer=ZO_OPT_ADAM, gamma_out=None):
    """losses: a CUDA fp32 tensor, or a CPU fp32 tensor / numpy array (copied by the library
    on the context's stream; a page-locked CPU tensor is read only when the stream reaches
    that copy, so keep it alive and unchanged until then)."""
    import numpy as np
    keep = None
    if hasattr(losses, "is_cuda") and losses.is_cuda:
        ptr, n, on_host = _ptr(losses), losses.numel(), 0
    else:
        keep = np.ascontiguousarray(np.asarray(losses, dtype=np.float32))
        ptr, n, on_host = keep.ctypes.data, keep.size, 1
    _check(LIB.zo_step(ctx, int(t), int(adam_t), ptr, int(n), on_host, int(scheme), int(optimizer),
                       float(eps), float(lr), float(beta1), float(beta2), float(eps_adam),
                       int(restore_query), float(restore_coef), _ptr(gamma_out)), "zo_step")
    del keep


def zo_mezo_perturb(ctx, t, coef):
    _check(LIB.zo_mezo_perturb(ctx, int(t), float(coef)), "zo_mezo_perturb")


def zo_linear_prepare(ctx, t, qa, ca, qb, cb, eps):
    """C_i = eps (ca Z_qa + cb Z_qb) at step t and P_i = C_i V_i^T for every matrix, for the
    zo_linear_perturbed calls of one loss evaluation."""
    _check(LIB.zo_linear_prepare(ctx, int(t), int(qa), float(ca), int(qb), float(cb),
                                 float(eps)), "zo_linear_prepare")


def zo_linear_perturbed(ctx, i, X, Y):
    """Y = X (W_i + U_i C_i V_i^T)^T with the prepared C_i; X (T x n) and Y (T x m) bf16
    CUDA tensors with unit column stride."""
    if X.dim() != 2 or Y.dim() != 2 or X.stride(1) != 1 or Y.stride(1) != 1 or X.shape[0] != Y.shape[0]:
        raise ValueError("X and Y must be 2-D, row-major (unit column stride), with the same rows")
    _check(LIB.zo_linear_perturbed(ctx, int(i), _ptr(X), int(X.shape[0]), int(X.stride(0)),
                                   _ptr(Y), int(Y.stride(0))), "zo_linear_perturbed")


def zo_sync_status(ctx):
    _check(LIB.zo_sync_status(ctx), "zo_sync_status")


def zo_set_option(ctx, option, value):
    _check(LIB.zo_set_option(ctx, int(option), int(value)), "zo_set_option")


def zo_get_timing(ctx):
    ms = ctypes.c_double()
    n = ctypes.c_int64()
    _check(LIB.zo_get_timing(ctx, ctypes.byref(ms), ctypes.byref(n)), "zo_get_timing")
    return ms.value, n.value


def zo_wpass_path(ctx):
    return int(LIB.zo_wpass_path(ctx))


def zo_linear_tiling(ctx):
    return int(LIB.zo_linear_tiling(ctx))


def zo_kernel_launches(ctx):
    return int(LIB.zo_kernel_launches(ctx))


def zo_perturb_noalloc(W, U, V, r, seed, matrix_index, t, qa, ca, qb, cb, eps, stream=None):
    """One perturbation pass on one matrix with no device allocation (see include/zo.h).
    W: m x n bf16/fp32 with unit column stride; U (m x r) and V (n x r) contiguous fp32 --
    checked here, since the C ABI cannot see the sizes behind its pointers."""
    import torch
    if W.dtype == torch.bfloat16:
        dt = ZO_BF16
    elif W.dtype == torch.float32:
        dt = ZO_F32
    else:
        raise ZoError(ZO_ERR_DTYPE, "zo_perturb_noalloc", str(W.dtype))
    if W.dim() != 2 or W.stride(1) != 1:
        raise ZoError(ZO_ERR_SHAPE, "zo_perturb_noalloc", "W must be 2-D with unit column stride")
    for name, t_, rows in (("U", U, W.shape[0]), ("V", V, W.shape[1])):
        if t_.dtype != torch.float32 or not t_.is_contiguous():
            raise ZoError(ZO_ERR_DTYPE, "zo_perturb_noalloc", f"{name} must be contiguous fp32")
        if tuple(t_.shape) != (rows, int(r)):
            raise ZoError(ZO_ERR_SHAPE, "zo_perturb_noalloc",
                          f"{name} has shape {tuple(t_.shape)}, expected {(rows, int(r))}")
    _check(LIB.zo_perturb_noalloc(_ptr(W), W.shape[0], W.shape[1], W.stride(0), dt, _ptr(U),
                                  _ptr(V), int(r), int(seed) & (2**64 - 1), int(matrix_index),
                                  int(t), int(qa), float(ca), int(qb), float(cb), float(eps),
                                  _stream_handle(stream)), "zo_perturb_noalloc")


def zo_philox_fill(seed, x1, x2, x3, out, stream=None):
    _check(LIB.zo_philox_fill(int(seed) & (2**64 - 1), int(x1), int(x2), int(x3), _ptr(out),
                              out.numel(), _stream_handle(stream)), "zo_philox_fill")


def zo_normal_fill(seed, x1, x2, x3, out, stream=None):
    _check(LIB.zo_normal_fill(int(seed) & (2**64 - 1), int(x1), int(x2), int(x3), _ptr(out),
                              out.numel(), _stream_handle(stream)), "zo_normal_fill")


def _code_of(dtype, where, name):
    import torch
    if dtype == torch.bfloat16:
        return ZO_BF16
    if dtype == torch.float32:
        return ZO_F32
    raise ZoError(ZO_ERR_DTYPE, where, f"{name} is {dtype}: bf16 or fp32")


def _dtype_code(t, where, name):
    return _code_of(t.dtype, where, name)


def _rows(t, where, name, shape, dtype, device):
    """(pointer, row stride) of a rows x cols matrix with unit column stride (None -> NULL)."""
    if t is None:
        return None, 0
    size = t.shape
    if len(size) != 2 or (shape is not None and size != shape):
        raise ZoError(ZO_ERR_SHAPE, where, f"{name} has shape {tuple(size)}, "
                                           f"expected {'2-D' if shape is None else tuple(shape)}")
    if not t.is_contiguous():
        rows, cols = size
        ld, step = t.stride()
        if (cols > 1 and step != 1) or (rows > 1 and ld < cols):
            raise ZoError(ZO_ERR_SHAPE, where, f"{name} needs unit column stride and separate rows")
    else:
        rows, ld = 2, size[1]
    if dtype is not None and t.dtype != dtype:
        raise ZoError(ZO_ERR_DTYPE, where, f"{name} is {t.dtype}, expected {dtype}")
    if device is not None and t.device != device:
        raise ZoError(ZO_ERR_INVALID_ARG, where, f"{name} is on {t.device}, expected {device}")
    return t.data_ptr(), ld if rows > 1 else size[1]


def _on_device(t, where):
    if not t.is_cuda:
        raise ZoError(ZO_ERR_INVALID_ARG, where, f"the tensors are on {t.device}, not on a GPU")


def _vector(t, where, name, n, dtype, device):
    """Pointer of a contiguous vector of n values (None -> NULL)."""
    if t is None:
        return None
    size = t.shape
    if len(size) != 1 or size[0] != n or not t.is_contiguous():
        raise ZoError(ZO_ERR_SHAPE, where, f"{name} must be a contiguous vector of {n} values")
    if t.dtype != dtype:
        raise ZoError(ZO_ERR_DTYPE, where, f"{name} is {t.dtype}, expected {dtype}")
    if t.device != device:
        raise ZoError(ZO_ERR_INVALID_ARG, where, f"{name} is on {t.device}, expected {device}")
    return t.data_ptr()


def zo_layernorm_forward(X, R, weight, bias, eps, Y, H=None, mean=None, rstd=None, stream=None):
    """Y = LayerNorm(X (+ R)) row by row (see include/zo.h); every tensor is checked here,
    since the C ABI cannot see the sizes behind its pointers."""
    import torch
    at = "zo_layernorm_forward"
    px, ldx = _rows(X, at, "X", None, None, None)
    shape, dt, dev = X.shape, X.dtype, X.device
    code, n = _dtype_code(X, at, "X"), X.shape[1]
    w = weight if weight is not None else bias
    wdt = torch.float32 if w is None else w.dtype
    wcode = ZO_F32 if w is None else _dtype_code(w, at, "weight")
    pr, ldr = _rows(R, at, "R", shape, dt, dev)
    py, ldy = _rows(Y, at, "Y", shape, dt, dev)
    ph, ldh = _rows(H, at, "H", shape, dt, dev)
    _on_device(X, at)
    _check(LIB.zo_layernorm_forward(
        px, ldx, pr, ldr, shape[0], n, code, _vector(weight, at, "weight", n, wdt, dev),
        _vector(bias, at, "bias", n, wdt, dev), wcode, float(eps), py, ldy, ph, ldh,
        _vector(mean, at, "mean", shape[0], torch.float32, dev),
        _vector(rstd, at, "rstd", shape[0], torch.float32, dev), _stream_handle(stream)), at)


def zo_layernorm_workspace(rows, cols):
    """Bytes of workspace that zo_layernorm_backward needs for its column sums."""
    return int(LIB.zo_layernorm_workspace(int(rows), int(cols)))


def zo_layernorm_backward(dY, X, dR, weight, mean, rstd, dX, dweight=None, dbias=None,
                          workspace=None, stream=None):
    """dX, dweight and dbias of zo_layernorm_forward (see include/zo.h).  workspace: a
    contiguous uint8 tensor of zo_layernorm_workspace(rows, cols) bytes."""
    import torch
    at = "zo_layernorm_backward"
    px, ldx = _rows(X, at, "X", None, None, None)
    shape, dt, dev = X.shape, X.dtype, X.device
    code, (rows, n) = _dtype_code(X, at, "X"), X.shape
    w = weight if weight is not None else dweight if dweight is not None else dbias
    wdt = torch.float32 if w is None else w.dtype
    wcode = ZO_F32 if w is None else _dtype_code(w, at, "weight")
    pdy, lddy = _rows(dY, at, "dY", shape, dt, dev)
    pdr, lddr = _rows(dR, at, "dR", shape, dt, dev)
    pdx, lddx = _rows(dX, at, "dX", shape, dt, dev)
    ws, ws_bytes = None, 0
    if workspace is not None:
        if workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != dev:
            raise ZoError(ZO_ERR_INVALID_ARG, at, "workspace must be contiguous uint8 beside X")
        ws, ws_bytes = workspace.data_ptr(), workspace.numel()
    _on_device(X, at)
    _check(LIB.zo_layernorm_backward(
        pdy, lddy, px, ldx, pdr, lddr, rows, n, code, _vector(weight, at, "weight", n, wdt, dev),
        wcode, _vector(mean, at, "mean", rows, torch.float32, dev),
        _vector(rstd, at, "rstd", rows, torch.float32, dev), pdx, lddx,
        _vector(dweight, at, "dweight", n, wdt, dev), _vector(dbias, at, "dbias", n, wdt, dev),
        ws, ws_bytes, _stream_handle(stream)), at)


def zo_layernorm_sync_status(stream=None):
    _check(LIB.zo_layernorm_sync_status(_stream_handle(stream)), "zo_layernorm_sync_status")


def make_muon_matrix(W, G, M=None):
    """zo_muon_matrix for torch tensors: W and G m x n (bf16 or fp32, any row stride), M a
    contiguous m x n fp32 momentum or None."""
    import torch
    at = "make_muon_matrix"
    pw, ldw = _rows(W, at, "W", None, None, None)
    pg, ldg = _rows(G, at, "G", W.shape, None, W.device)
    if M is not None and (tuple(M.shape) != tuple(W.shape) or not M.is_contiguous()):
        raise ZoError(ZO_ERR_SHAPE, at, "M must be contiguous with W's shape")
    if M is not None and (M.dtype != torch.float32 or M.device != W.device):
        raise ZoError(ZO_ERR_DTYPE, at, "M must be fp32 beside W")
    _on_device(W, at)
    return zo_muon_matrix(pw, pg, _ptr(M), W.shape[0], W.shape[1], ldw, ldg,
                          _dtype_code(W, at, "W"), _dtype_code(G, at, "G"))


def _coeffs(steps, coeffs, where):
    """(steps, address, keep-alive) of a sequence of (a, b, c) per step, or of the default."""
    import numpy as np
    if coeffs is None:
        return int(steps), None, None
    arr = np.ascontiguousarray(np.asarray(coeffs, dtype=np.float32))
    if arr.shape != (int(steps), 3):
        raise ZoError(ZO_ERR_SHAPE, where, f"coeffs has shape {arr.shape}, expected {(steps, 3)}")
    return int(steps), arr.ctypes.data, arr


def zo_muon_workspace(mats):
    """Bytes of device workspace for a context over `mats`."""
    arr = (zo_muon_matrix * len(mats))(*mats)
    n = int(LIB.zo_muon_workspace(arr, len(mats)))
    if n <= 0:
        raise ZoError(ZO_ERR_INVALID_ARG, "zo_muon_workspace", zo_last_error())
    return n


def zo_muon_create(mats, workspace, stream=None):
    arr = (zo_muon_matrix * len(mats))(*mats)
    ctx = ctypes.c_void_p()
    _check(LIB.zo_muon_create(ctypes.byref(ctx), arr, len(mats), _ptr(workspace),
                              workspace.numel() * workspace.element_size(),
                              _stream_handle(stream)), "zo_muon_create")
    return ctx


def zo_muon_destroy(ctx):
    _check(LIB.zo_muon_destroy(ctx), "zo_muon_destroy")


def zo_orthogonalize(ctx, steps=5, coeffs=None, eps=1e-7):
    n, ptr, keep = _coeffs(steps, coeffs, "zo_orthogonalize")
    _check(LIB.zo_orthogonalize(ctx, n, ptr, float(eps)), "zo_orthogonalize")
    del keep


def zo_muon_step(ctx, momentum, nesterov, lr, weight_decay, adjust, steps=5, coeffs=None,
                 eps=1e-7):
    n, ptr, keep = _coeffs(steps, coeffs, "zo_muon_step")
    _check(LIB.zo_muon_step(ctx, float(momentum), int(bool(nesterov)), float(lr),
                            float(weight_decay), int(adjust), n, ptr, float(eps)), "zo_muon_step")
    del keep


def zo_muon_sync_status(ctx):
    _check(LIB.zo_muon_sync_status(ctx), "zo_muon_sync_status")


def zo_muon_launches(ctx):
    return int(LIB.zo_muon_launches(ctx))
