"""The preference loss's entry points refuse bad arguments on the host (no GPU needed)."""

import pytest
import torch

FORWARD = dict(x=0x1000, ldl=100, rows=6, vocab=100, dtype=1, labels=0x2000, offsets=0x3000, pairs=1,
               ref=0, kind=0, beta=0.1, smoothing=0.0, margin=0.0, average=0, loss=0x4000,
               losses=0x5000, logps=0x6000, lse=0, dlogp=0, ws=0x10000, ws_bytes=1 << 30, stream=0)
BACKWARD = dict(x=0x1000, ldl=100, rows=6, vocab=100, dtype=1, labels=0x2000, lse=0x3000,
                dlogp=0x4000, dloss=0, out=0x8000, ldd=100, stream=0)


def _call(fn, base, kw):
    args = dict(base)
    args.update(kw)
    assert set(args) == set(base)
    return fn(*[None if v == 0 and k in ("x", "labels", "offsets", "ref", "loss", "losses", "logps",
                                         "lse", "dlogp", "ws", "dloss", "out", "stream") else v
                for k, v in args.items()])


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), 4), (dict(rows=-1), 2), (dict(vocab=0), 2), (dict(ldl=99), 2),
    (dict(rows=1 << 26), 2), (dict(pairs=0), 2), (dict(kind=3), 1), (dict(kind=-1), 1),
    (dict(beta=0.0), 1), (dict(beta=float("nan")), 1), (dict(margin=float("inf")), 1),
    (dict(smoothing=0.5), 1), (dict(smoothing=-0.1), 1), (dict(smoothing=0.1, kind=1), 1),
    (dict(margin=1.0, kind=2), 1), (dict(x=0), 1), (dict(labels=0), 1), (dict(offsets=0), 1),
    (dict(loss=0), 1), (dict(losses=0), 1), (dict(logps=0), 1), (dict(ws=0), 1),
    (dict(ws_bytes=100), 1), (dict(x=0x1001), 3), (dict(x=0x1002, dtype=0), 3),
    (dict(labels=0x2004), 3), (dict(loss=0x4002), 3), (dict(ws=0x10008), 3)])
def test_forward_refuses(lib, kw, status):
    assert _call(lib.LIB.zo_preference_forward, FORWARD, kw) == status and lib.zo_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), 4), (dict(ldd=99), 2), (dict(vocab=0), 2), (dict(x=0), 1), (dict(labels=0), 1),
    (dict(lse=0), 1), (dict(dlogp=0), 1), (dict(out=0), 1), (dict(out=0x8001), 3),
    (dict(out=0x1000, ldd=104), 1), (dict(dloss=0x9002), 3)])
def test_backward_refuses(lib, kw, status):
    assert _call(lib.LIB.zo_preference_backward, BACKWARD, kw) == status and lib.zo_last_error()


def test_no_rows_are_no_work(lib):
    assert _call(lib.LIB.zo_preference_backward, BACKWARD, dict(rows=0, x=0, out=0)) == lib.ZO_OK


def test_workspace_covers_parts_for_any_number_of_sms(lib):
    ws = lib.LIB.zo_preference_workspace
    assert ws(-1, 10) == 0 and ws(4, 0) == 0
    assert ws(0, 10) == 256 and ws(1, 10) == 512
    assert ws(1, 128000) >= 512 + 8 * 16
    assert ws(100000, 32000) == 256 + 400128


def test_binding_and_helpers_refuse_what_the_abi_cannot_see(lib):
    from paper_2608_15665_gb300 import firstorder as fo
    x, labels = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int64)
    offsets = torch.tensor([0, 2, 4])
    good = dict(logits=x, labels=labels, offsets=offsets)
    for kw in (dict(logits=x.half()), dict(logits=x.t()), dict(labels=labels.int()),
               dict(labels=labels[:3]), dict(offsets=offsets[:2]), dict(offsets=offsets.int()),
               dict(ref_logps=torch.zeros(3)), dict(ref_logps=torch.zeros(2).double()),
               dict(kind="other"), dict(out=torch.zeros(2)), dict(logits=x.clone().requires_grad_()),
               {}):                                                       # {}: not on a GPU
        with pytest.raises(lib.ZoError):
            fo.preference_loss(**{**good, **kw})
    f = torch.zeros(4)
    good = dict(logits=x, labels=labels, lse=f, dlogp=f)
    for kw in (dict(lse=f[:3]), dict(dlogp=f.double()), dict(dloss=torch.zeros(2)),
               dict(out=torch.zeros(4, 9)), dict(out=x.bfloat16()), {}):
        with pytest.raises(lib.ZoError):
            fo.preference_loss_backward(**{**good, **kw})
    args = dict(logits=x, labels=labels, offsets=offsets, ref_logps=None, kind=0, beta=0.1,
                smoothing=0.0, margin=0.0, average=False, loss=torch.zeros(()),
                losses=torch.zeros(1), logps=torch.zeros(2),
                workspace=torch.zeros(4096, dtype=torch.uint8))
    for kw in (dict(losses=torch.zeros(2)), dict(logps=torch.zeros(1)), dict(workspace=None),
               dict(lse=torch.zeros(3)), dict(loss=torch.zeros(2)), {}):
        with pytest.raises(lib.ZoError):
            lib.zo_preference_forward(**{**args, **kw})
    for kw in (dict(dlogits=x[:3]), {}):
        with pytest.raises(lib.ZoError):
            lib.zo_preference_backward(**{**dict(logits=x, labels=labels, lse=f, dlogp=f, dloss=None,
                                                 dlogits=x), **kw})


def test_a_step_takes_losses_as_numbers_and_does_not_touch_them(lib, monkeypatch):
    from paper_2608_15665_gb300 import schedule
    seen = []
    monkeypatch.setattr(lib, "zo_step", lambda ctx, t, adam_t, losses, *a: seen.append(losses))
    z = object.__new__(schedule.SubZeroPlus)
    z.ctx = None
    losses = [1.0, 2.0]
    z.step(0, 1, losses, "central", 1e-3, 1e-3, 0.9, 0.95, 1e-8, -1, 0.0)
    assert seen[0] is losses
