"""Layer normalisation's entry points refuse bad arguments on the host, before anything is
launched (no GPU needed)."""

import pytest
import torch


def _fwd(lib, X=0x1000, ldx=64, R=None, ldr=0, rows=4, cols=64, dtype=1, w=0x2000, b=0x3000,
         wdtype=1, eps=1e-5, Y=0x4000, ldy=64, H=None, ldh=0, mean=0x5000, rstd=0x6000):
    return lib.LIB.zo_layernorm_forward(X, ldx, R, ldr, rows, cols, dtype, w, b, wdtype, eps, Y,
                                        ldy, H, ldh, mean, rstd, None)


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), 1), (dict(Y=None), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
    (dict(eps=float("inf")), 1),
    (dict(R=0x7000, ldr=64), 1), (dict(H=0x7000, ldh=64), 1),       # residual without sum, sum alone
    (dict(dtype=2), 4), (dict(wdtype=-1), 4),
    (dict(rows=-1), 2), (dict(cols=0), 2), (dict(rows=2**31), 2), (dict(cols=2**31), 2),
    (dict(ldx=63), 2), (dict(ldy=63), 2), (dict(R=0x7000, ldr=63, H=0x8000, ldh=64), 2),
    (dict(X=0x1001), 3), (dict(w=0x2001), 3), (dict(mean=0x5002), 3), (dict(Y=0x4002, dtype=0), 3),
])
def test_forward_refuses(lib, kw, status):
    assert _fwd(lib, **kw) == status


def _bwd(lib, dY=0x1000, lddy=64, X=0x2000, ldx=64, dR=None, lddr=0, rows=4, cols=64, dtype=1,
         w=0x3000, wdtype=1, mean=0x4000, rstd=0x5000, dX=0x6000, lddx=64, dw=0x7000, db=0x8000,
         ws=0x9000, n=0):
    return lib.LIB.zo_layernorm_backward(dY, lddy, X, ldx, dR, lddr, rows, cols, dtype, w, wdtype,
                                         mean, rstd, dX, lddx, dw, db, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dY=None), 1), (dict(X=None), 1), (dict(mean=None), 1), (dict(rstd=None), 1),
    (dict(dX=None), 1), (dict(dtype=3), 4), (dict(wdtype=5), 4),
    (dict(rows=-2), 2), (dict(cols=0), 2), (dict(lddy=10), 2), (dict(lddx=10), 2),
    (dict(dR=0xA000, lddr=3), 2), (dict(dX=0x6001), 3), (dict(ws=0x9008), 3),
])
def test_backward_refuses(lib, kw, status):
    assert _bwd(lib, **kw) == status


def test_no_rows_launch_nothing(lib):
    assert _fwd(lib, rows=0, X=None, Y=None) == lib.ZO_OK
    assert _bwd(lib, rows=0, dw=None, db=None) == lib.ZO_OK
    assert lib.zo_layernorm_workspace(0, 64) == 0


def test_binding_refuses_what_the_abi_cannot_see(lib):
    x, v = torch.zeros(4, 8), torch.zeros(8)
    out = torch.zeros(4, 8)
    bad = [
        dict(X=torch.zeros(8, 4).t()), dict(Y=torch.zeros(4, 7)), dict(weight=torch.zeros(7)),
        dict(weight=torch.zeros(16)[::2]), dict(Y=out.double()), dict(X=x.half()),
        dict(bias=v.to(torch.bfloat16)), dict(mean=torch.zeros(3)), dict(X=torch.zeros(4)),
        dict(X=torch.zeros(1, 8).expand(4, 8)),
    ]
    for kw in bad:
        args = dict(X=x, R=None, weight=v, bias=v, eps=1e-5, Y=out, mean=None)
        args.update(kw)
        with pytest.raises(lib.ZoError):
            lib.zo_layernorm_forward(**args)
    with pytest.raises(lib.ZoError):
        lib.zo_layernorm_backward(out, x, None, v, torch.zeros(4), torch.zeros(4), out, v, v,
                                  torch.zeros(64))                 # workspace not uint8
