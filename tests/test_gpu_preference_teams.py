"""The preference loss around the widths where rows pass from warps to CTAs and from one part to
several, with few rows and with as many as fill a GB300's SMs twice, in memory that holds NaN before
the call: every row is summed whole, and what is written is all there is.

Tolerances: a row's sum goes over 32 threads at least, each with two running sums, so V / 64 + 60
roundings of it; the rest as for wider rows (a term is off by 2^-22 and by two roundings of its
exponent)."""

import numpy as np
import pytest
import torch

from test_gpu_preference import U, TYPES, check_gradient, f64

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.mark.parametrize("rows", [2, 3, 5, 100, 160, 303, 304])
@pytest.mark.parametrize("dtype,vocab", [
    ("bf16", 8184), ("bf16", 8191), ("bf16", 8192), ("bf16", 8193), ("bf16", 8200), ("bf16", 4096),
    ("bf16", 4104), ("bf16", 16384), ("f32", 4088), ("f32", 4095), ("f32", 4096), ("f32", 4097),
    ("f32", 4104), ("f32", 2048), ("f32", 2056), ("f32", 8192)])
def test_rows_at_the_borders_of_the_teams(lib, gpu, dtype, vocab, rows):
    g = torch.Generator().manual_seed(rows * vocab)
    x = (torch.randn(rows, vocab, generator=g) * 3.0).to(TYPES[dtype]).to(gpu)
    labels = torch.randint(0, vocab, (rows,), generator=g)
    labels[rows // 2] = -100
    labels = labels.to(gpu)
    first = max(1, rows // 3)
    offsets = torch.tensor([0, first, rows if rows < 5 else rows - 1], device=gpu)
    loss = torch.full((), NAN, device=gpu)
    losses, logps = torch.full((1,), NAN, device=gpu), torch.full((2,), NAN, device=gpu)
    lse, dlogp = torch.full((rows,), NAN, device=gpu), torch.full((rows,), NAN, device=gpu)
    n = lib.zo_preference_workspace(rows, vocab)
    ws = torch.full((-(-n // 4),), NAN, device=gpu).view(torch.uint8)[:n]
    s = torch.cuda.current_stream()
    lib.zo_preference_forward(x, labels, offsets, None, lib.ZO_PREFERENCE_SIGMOID, 0.5, 0.0, 0.0, False,
                              loss, losses, logps, lse, dlogp, ws, stream=s)
    xs, ls, end = f64(x), labels.cpu().numpy(), int(offsets[2])
    top = xs.max(1, keepdims=True)
    e = np.exp(xs - top)
    total = e.sum(1)
    want = top[:, 0] + np.log(total)
    err = (vocab / 64 + 64) * U + 2 * U * (e * np.abs(xs - top)).sum(1) / total
    counted = (ls >= 0) & (np.arange(rows) < end)
    got = f64(lse)
    assert np.all(np.abs(got - want)[counted] <= (err + U * np.abs(want))[counted])
    assert np.all(got[~counted] == 0) and np.all(f64(dlogp)[~counted] == 0)
    logp = np.where(counted, xs[np.arange(rows), np.maximum(ls, 0)] - want, 0.0)
    per = np.where(counted, err + 2 * U * np.abs(logp), 0.0)
    sums = np.array([logp[:first].sum(), logp[first:end].sum()])
    lim = np.array([per[:first].sum(), per[first:end].sum()])
    assert np.all(np.abs(f64(logps) - sums) <= lim + U * np.abs(sums))
    z, zerr = 0.5 * (sums[0] - sums[1]), 0.5 * lim.sum()
    assert abs(float(loss) - np.logaddexp(0.0, -z)) <= zerr + 8 * U * (np.logaddexp(0.0, -z) + 1)
    assert float(losses[0]) == float(loss)
    slope = -0.5 * np.exp(-np.logaddexp(0.0, z))
    sign = np.where(np.arange(rows) < first, 1.0, -1.0) * counted
    assert np.all(np.abs(f64(dlogp) - sign * slope) <= 0.125 * zerr + 8 * U * 0.5 + 4 * U * abs(slope))
    d = torch.full_like(x, NAN)
    lib.zo_preference_backward(x, labels, lse, dlogp, None, d, stream=s)
    check_gradient(d, xs, ls, f64(lse), f64(dlogp), 1.0, dtype)
