"""AdamW's entry points refuse bad arguments on the host (no GPU needed)."""

import ctypes

import pytest
import torch


def _tensor(lib, W=0x1000, G=0x2000, M=0x3000, V=0x4000, Em=0x5000, Ev=0x6000, m=64, n=96, ldw=96,
            ldg=96, dtype=1, gd=1):
    return lib.zo_adamw_tensor(W, G, M, V, Em, Ev, m, n, ldw, ldg, dtype, gd)


def _other(lib, **kw):
    args = dict(W=0x11000, G=0x12000, M=0x13000, V=0x14000, Em=0x15000, Ev=0x16000)
    args.update(kw)
    return _tensor(lib, **args)


def _arr(lib, *tensors):
    return (lib.zo_adamw_tensor * len(tensors))(*tensors)


BAD = [
    (dict(W=0), 1), (dict(G=0), 1), (dict(M=0), 1), (dict(V=0), 1), (dict(Em=0), 1),
    (dict(Ev=0), 1), (dict(dtype=2), 4), (dict(gd=-1), 4), (dict(m=-1), 2), (dict(n=-1), 2),
    (dict(ldw=95), 2), (dict(ldg=95), 2), (dict(m=1 << 18, n=1 << 17, ldw=1 << 17, ldg=1 << 17), 2),
    (dict(W=0x11001), 3), (dict(G=0x12001), 3), (dict(G=0x12002, gd=0), 3),
]


@pytest.mark.parametrize("kw,status", BAD)
def test_create_and_workspace_refuse(lib, kw, status):
    arr = _arr(lib, _tensor(lib), _other(lib, **kw))
    ctx = ctypes.c_void_p(7)
    assert lib.LIB.zo_adamw_workspace(arr, 2, 8) == 0
    assert lib.LIB.zo_adamw_create(ctypes.byref(ctx), arr, 2, 8, 0, 0x100000, 1 << 40, None) == status
    assert not ctx.value and lib.zo_last_error()


def test_states_of_32_bits_need_no_exponents_but_their_alignment(lib):
    assert lib.LIB.zo_adamw_workspace(_arr(lib, _other(lib, Em=0, Ev=0)), 1, 32) > 0
    assert lib.LIB.zo_adamw_workspace(_arr(lib, _other(lib, M=0x13002)), 1, 32) == 0
    assert lib.LIB.zo_adamw_workspace(_arr(lib, _other(lib, M=0x13001)), 1, 8) > 0
    assert lib.LIB.zo_adamw_workspace(_arr(lib, _other(lib)), 1, 16) == 0


def test_a_missing_small_or_misaligned_workspace_is_refused(lib):
    arr = _arr(lib, _tensor(lib))
    need = lib.LIB.zo_adamw_workspace(arr, 1, 32)
    assert need > 0
    ctx = ctypes.c_void_p()
    create = lib.LIB.zo_adamw_create
    assert create(ctypes.byref(ctx), arr, 1, 32, 0, None, need, None) == lib.ZO_ERR_INVALID_ARG
    assert create(ctypes.byref(ctx), arr, 1, 32, 0, 0x100000, need - 1, None) == lib.ZO_ERR_INVALID_ARG
    assert create(ctypes.byref(ctx), arr, 1, 32, 0, 0x100080, need, None) == lib.ZO_ERR_ALIGN
    assert create(ctypes.byref(ctx), arr, 1, 16, 0, 0x100000, need, None) == lib.ZO_ERR_UNSUPPORTED
    assert create(None, arr, 1, 32, 0, 0x100000, need, None) == lib.ZO_ERR_INVALID_ARG
    assert create(ctypes.byref(ctx), arr, 0, 32, 0, 0x100000, need, None) == lib.ZO_ERR_INVALID_ARG
    assert lib.LIB.zo_adamw_workspace(None, 1, 32) == 0


@pytest.mark.parametrize("kw", [dict(W=0x1000), dict(M=0x3000), dict(V=0x3000), dict(Ev=0x5000)])
def test_a_buffer_that_a_step_writes_is_given_once(lib, kw):
    arr = _arr(lib, _tensor(lib), _other(lib, **kw))
    ctx = ctypes.c_void_p()
    create = lib.LIB.zo_adamw_create
    assert create(ctypes.byref(ctx), arr, 2, 8, 0, 0x100000, 1 << 40, None) == lib.ZO_ERR_INVALID_ARG
    assert "twice" in lib.zo_last_error()


def test_calls_on_a_null_context_are_refused(lib):
    L = lib.LIB
    assert L.zo_adamw_step(None, 1, None, 0.1, 0.9, 0.99, 1e-8, 0.0) == lib.ZO_ERR_INVALID_ARG
    assert L.zo_adamw_destroy(None) == lib.ZO_OK and L.zo_adamw_launches(None) == 0


def test_binding_refuses_what_the_abi_cannot_see(lib):
    W, s = torch.zeros(4, 8), torch.zeros(32)
    codes, e = torch.zeros(32, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8)
    for kw in (dict(G=torch.zeros(4, 7)), dict(G=torch.zeros(8, 4).t()), dict(W=W.half()),
               dict(G=W.double()), dict(M=torch.zeros(31)), dict(V=torch.zeros(64)[::2]),
               dict(M=s.bfloat16()), dict(M=codes), dict(Em=e), dict(M=codes, V=codes, Ev=e),
               dict(M=codes, V=codes, Em=e, Ev=torch.zeros(2, dtype=torch.uint8)),
               dict(M=s, V=s, Em=e, Ev=e), dict(W=W[:, ::2], G=W[:, ::2]),
               dict(W=torch.zeros(64)[::2], G=torch.zeros(64)[::2]), {}):   # {}: not on a GPU
        args = dict(W=W, G=W, M=s, V=s)
        args.update(kw)
        with pytest.raises(lib.ZoError):
            lib.make_adamw_tensor(**args)


def test_handle_refuses(lib):
    from paper_2608_15665_gb300 import firstorder as fo
    W = [torch.zeros(4)]
    for kw in (dict(weights=[]), dict(bits=16), dict(states=[fo.adamw_state(W[0], 8)]),
               dict(states=[fo.adamw_state(W[0])], bits=8), dict(count=torch.zeros(1)),
               dict(count=torch.zeros(2, dtype=torch.int64)), {}):          # {}: not on a GPU
        args = dict(weights=W)
        args.update(kw)
        with pytest.raises(lib.ZoError):
            fo.AdamW(**args)
    with pytest.raises(ValueError):
        fo.AdamW(W, grads=[])
    with pytest.raises(lib.ZoError):
        fo.adamw_state(W[0], 16)
