"""The orthogonalisation's entry points refuse bad arguments on the host (no GPU needed)."""

import ctypes

import numpy as np
import pytest
import torch


def _mat(lib, W=0x1000, G=0x2000, M=0x3000, m=64, n=96, ldw=96, ldg=96, dtype=1, gd=1):
    return lib.zo_muon_matrix(W, G, M, m, n, ldw, ldg, dtype, gd)


def _arr(lib, *mats):
    return (lib.zo_muon_matrix * len(mats))(*mats)


BAD = [
    (dict(W=0), 1), (dict(G=0), 1), (dict(dtype=2), 4), (dict(gd=-1), 4),
    (dict(m=0), 2), (dict(n=0), 2), (dict(ldw=95), 2), (dict(ldg=95), 2), (dict(m=1 << 24), 2),
    (dict(m=70000, n=70000, ldw=70000, ldg=70000), 2),           # min(m, n) > 2^16
    (dict(W=0x1001), 3), (dict(G=0x2001), 3), (dict(M=0x3002), 3), (dict(G=0x2002, gd=0), 3),
]


@pytest.mark.parametrize("kw,status", BAD)
def test_create_and_workspace_refuse(lib, kw, status):
    arr = _arr(lib, _mat(lib), _mat(lib, **kw))
    ctx = ctypes.c_void_p(7)
    assert lib.LIB.zo_muon_workspace(arr, 2) == 0
    assert lib.LIB.zo_muon_create(ctypes.byref(ctx), arr, 2, 0x10000, 1 << 40, None) == status
    assert not ctx.value and lib.zo_last_error()


def test_a_missing_small_or_misaligned_workspace_is_refused(lib):
    arr = _arr(lib, _mat(lib))
    need = lib.LIB.zo_muon_workspace(arr, 1)
    assert need > 0
    ctx = ctypes.c_void_p()
    create = lib.LIB.zo_muon_create
    assert create(ctypes.byref(ctx), arr, 1, None, need, None) == lib.ZO_ERR_INVALID_ARG
    assert create(ctypes.byref(ctx), arr, 1, 0x10000, need - 1, None) == lib.ZO_ERR_INVALID_ARG
    assert create(ctypes.byref(ctx), arr, 1, 0x10080, need, None) == lib.ZO_ERR_ALIGN
    assert create(None, arr, 1, 0x10000, need, None) == lib.ZO_ERR_INVALID_ARG
    assert create(ctypes.byref(ctx), arr, 0, 0x10000, need, None) == lib.ZO_ERR_INVALID_ARG
    assert lib.LIB.zo_muon_workspace(None, 1) == 0


def test_groups_share_their_buffers(lib):
    one = lib.LIB.zo_muon_workspace(_arr(lib, _mat(lib, m=8192, n=8192, ldw=8192, ldg=8192)), 1)
    many = lib.LIB.zo_muon_workspace(
        _arr(lib, *[_mat(lib, m=8192, n=8192, ldw=8192, ldg=8192)] * 40), 40)
    assert many < 3 * one


def test_calls_on_a_null_context_are_refused(lib):
    L = lib.LIB
    assert L.zo_orthogonalize(None, 5, None, 1e-7) == lib.ZO_ERR_INVALID_ARG
    assert L.zo_muon_step(None, 0.9, 1, 0.1, 0.0, 0, 5, None, 1e-7) == lib.ZO_ERR_INVALID_ARG
    assert L.zo_muon_sync_status(None) == lib.ZO_ERR_INVALID_ARG
    assert L.zo_muon_destroy(None) == lib.ZO_OK and L.zo_muon_launches(None) == 0


def test_binding_refuses_what_the_abi_cannot_see(lib):
    W = torch.zeros(4, 8)
    for kw in (dict(G=torch.zeros(4, 7)), dict(G=torch.zeros(8, 4).t()), dict(W=W.half()),
               dict(G=W.double()), dict(M=torch.zeros(4, 8, dtype=torch.bfloat16)),
               dict(M=torch.zeros(4, 9)[:, :8]), dict(W=torch.zeros(8)),
               dict(W=torch.zeros(4, 1).expand(4, 8)), {}):          # {}: not on a GPU
        args = dict(W=W, G=W, M=None)
        args.update(kw)
        with pytest.raises(lib.ZoError):
            lib.make_muon_matrix(**args)
    with pytest.raises(lib.ZoError):
        lib._coeffs(5, np.zeros((4, 3)), "test")
