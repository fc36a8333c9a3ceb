"""The gated linear block's entry points refuse bad arguments on the host (no GPU needed)."""

import pytest
import torch

FORWARD = dict(X=0x1000, ldx=64, T=5, D=64, Wg=0x2000, ldwg=64, Wu=0x3000, ldwu=64, F=32, act=0,
               H=0x4000, ldh=32, G=0x5000, ldg=32, U=0x6000, ldu=32, stream=0)
BACKWARD = dict(dH=0x7000, lddh=32, X=0x1000, ldx=64, T=5, D=64, Wg=0x2000, ldwg=64, Wu=0x3000,
                ldwu=64, F=32, act=0, G=0x5000, ldg=32, U=0x6000, ldu=32, dX=0x8000, lddx=64,
                dWg=0x9000, lddwg=64, dWu=0xa000, lddwu=64, ws=0x10000, ws_bytes=1 << 30, stream=0)
POINTERS = ("X", "Wg", "Wu", "H", "G", "U", "dH", "dX", "dWg", "dWu", "ws", "stream")


def _call(fn, base, kw):
    args = dict(base)
    args.update(kw)
    assert set(args) == set(base)
    return fn(*[None if v == 0 and k in POINTERS else v for k, v in args.items()])


COMMON = [(dict(act=2), 1), (dict(act=-1), 1), (dict(T=-1), 2), (dict(T=1 << 24), 2), (dict(D=0), 2),
          (dict(D=60), 2), (dict(F=12), 2), (dict(F=1 << 24), 2),
          (dict(T=1 << 20, F=1 << 16, ldh=1 << 16, lddh=1 << 16), 2),
          (dict(D=1 << 20, F=1 << 18, ldx=1 << 20), 2), (dict(ldx=63), 2), (dict(ldwg=56), 2), (dict(ldx=68), 3), (dict(Wg=0x2008), 3),
          (dict(Wu=0), 1), (dict(ldu=24), 2)]


@pytest.mark.parametrize("kw,status", [(k, s) for k, s in COMMON if "lddh" not in k] + [
    (dict(G=0), 1), (dict(U=0), 1), (dict(X=0), 1), (dict(H=0), 1), (dict(H=0x4002), 3),
    (dict(ldh=36), 3)])
def test_forward_refuses(lib, kw, status):
    assert _call(lib.LIB.zo_gated_forward, FORWARD, kw) == status and lib.zo_last_error()


@pytest.mark.parametrize("kw,status", [(k, s) for k, s in COMMON if "lddh" not in k] + [
    (dict(dH=0), 1), (dict(G=0), 1), (dict(X=0), 1), (dict(dWg=0), 1), (dict(dWu=0), 1),
    (dict(ws=0), 1), (dict(ws_bytes=1535), 1), (dict(ws=0x10008), 3), (dict(dX=0x8008), 3),
    (dict(lddx=56), 2), (dict(lddwg=68), 3)])
def test_backward_refuses(lib, kw, status):
    assert _call(lib.LIB.zo_gated_backward, BACKWARD, kw) == status and lib.zo_last_error()


def test_no_tokens_and_nothing_wanted_are_no_work(lib):
    assert _call(lib.LIB.zo_gated_forward, FORWARD, dict(T=0, X=0, H=0, G=0, U=0)) == lib.ZO_OK
    assert _call(lib.LIB.zo_gated_backward, BACKWARD, dict(T=0, dWg=0, dWu=0)) == lib.ZO_OK
    assert _call(lib.LIB.zo_gated_backward, BACKWARD, dict(dX=0, dWg=0, dWu=0)) == lib.ZO_OK


def test_workspace(lib):
    ws = lib.LIB.zo_gated_workspace
    assert ws(0, 64, 64) == 0 and ws(5, 64, 32) == 2 * 768          # two rows a token
    assert ws(200, 64, 32) == 2 * 12800
    assert ws(5, 64, 33) == 0 and ws(-1, 8, 8) == 0 and ws(5, 60, 32) == 0
    assert ws(4096, 4096, 11008) == 2 * 2 * 4096 * 11008
    # a tile of dX whose K of 2 x 16 stages is split in four, and its counters
    assert ws(5, 64, 1024) == 2 * 2 * 5 * 1024 * 2 + 4 * 256 * 256 * 4 + 256


def test_binding_and_helpers_refuse_what_the_abi_cannot_see(lib):
    from paper_2608_15665_gb300 import firstorder as fo
    bf = torch.bfloat16
    x, w = torch.zeros(4, 16, dtype=bf), torch.zeros(24, 16, dtype=bf)
    h = torch.zeros(4, 24, dtype=bf)
    good = dict(x=x, w_gate=w, w_up=w)
    for kw in (dict(x=x.float()), dict(x=x[:, :8]), dict(w_up=w[:16]), dict(w_gate=w.t()),
               dict(x=x[0]), dict(act="relu"), dict(x=x.clone().requires_grad_()), {}):
        with pytest.raises(lib.ZoError):                             # {}: not on a GPU
            fo.gated_linear(**{**good, **kw})
        if "x" not in kw or not kw["x"].requires_grad:
            with pytest.raises(lib.ZoError):
                fo.gated_linear_backward(**{**dict(good, dh=h, gate=h, up=h), **kw})
    for kw in (dict(dh=h[:3]), dict(gate=h.float()), dict(up=h[:, :16])):
        with pytest.raises(lib.ZoError):
            fo.gated_linear_backward(**{**dict(good, dh=h, gate=h, up=h), **kw})
    for kw in (dict(H=h[:3]), dict(G=h.float(), U=h), dict(Wu=w[:8]), dict(Wg=w[:, :8]), {}):
        with pytest.raises(lib.ZoError):
            lib.zo_gated_forward(**{**dict(X=x, Wg=w, Wu=w, act=0, H=h), **kw})
    for kw in (dict(dX=h), dict(dWg=x), dict(workspace=h), dict(dH=x), {}):
        with pytest.raises(lib.ZoError):
            lib.zo_gated_backward(**{**dict(dH=h, X=x, Wg=w, Wu=w, act=0, G=h, U=h), **kw})
