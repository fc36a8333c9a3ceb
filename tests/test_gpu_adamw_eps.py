"""AdamW with an eps of nothing, or next to it: then the update is m / sqrt(v) down to the smallest
second moments that fp32 holds, v = 2^-149.

Tolerances as in test_gpu_adamw_range.py: the moments are fp32 arithmetic bit for bit, the update is off
by 24 u of itself (u = 2^-24), W by two roundings and half an ulp."""

import numpy as np
import pytest
import torch

from test_gpu_adamw import B1, B2, WD, f64, random_of, values
from test_gpu_adamw_range import check_w, codes_of, f, moments

pytestmark = pytest.mark.gpu


def gradients(n, low, high, seed, dev):
    """+-2^low .. 2^high"""
    g = torch.Generator().manual_seed(seed)
    size = 2.0 ** (torch.rand(n, generator=g, dtype=torch.float64) * (high - low) + low)
    return (torch.randn(n, generator=g).sign() * size).float().to(dev)


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-20, 1e-12, 1e-10, 1e-8])
@pytest.mark.parametrize("low,high", [(-68, -28), (-69, -60), (-20, 0)])
@pytest.mark.parametrize("bits,wide", [(32, True), (32, False), (8, True), (8, False)])
def test_steps_of_small_gradients(lib, gpu, bits, wide, low, high, eps):
    """wide: tensors on 16 bytes, else one element behind them."""
    from paper_2608_15665_gb300 import firstorder as fo
    n, lr, off = 20077, 1e-2, 0 if wide else 1
    g = torch.Generator().manual_seed(6)
    W = torch.zeros(n + off, device=gpu)[off:].copy_(torch.randn(n, generator=g) * 0.02)
    G = torch.zeros(n + off, device=gpu)[off:].copy_(gradients(n, low, high, 8, gpu))
    opt = fo.AdamW([W], [G], bits=bits, seed=4)
    s = opt.states[0]
    m, v = np.zeros(n, f), np.zeros(n, f)
    for t in (1, 2, 3):
        before, x = f64(W), f64(G).astype(f)
        if bits == 8:
            m, r = values(s.m, s.m_exp, (n,)), values(s.v, s.v_exp, (n,))
            m, v = moments(m, r, x, B2)
        else:
            m, v = f(B1) * m + f(1.0 - B1) * x, f(B2) * v + f(1.0 - B2) * (x * x)
        opt.step(lr, (B1, B2), eps, WD)
        torch.cuda.synchronize()
        # (a root in 8 bits is no less than its block's smallest code: only the first step sees the
        # squares alone)
        assert v.min() > 0 and (t > 1 or (v.min() < 2.0 ** -126) == (low < -60))
        check_w(W, before, m, v, t, lr, eps)
        if bits == 32:
            assert np.array_equal(f64(s.m), m) and np.array_equal(f64(s.v), v)
        elif eps < 1e-11:
            # and the codes are those of roots to nearest, whatever their size
            y, want = codes_of(np.sqrt(v).astype(np.float64), s.v_exp.cpu().numpy().astype(np.int64),
                               random_of(4, 0, t, n))
            assert np.array_equal(f64(s.v)[y >= 2.0 ** -6], want[y >= 2.0 ** -6])
    opt.close()


def test_squares_beyond_fp32_with_an_eps_of_nothing(lib, gpu):
    """As with any other eps: 32 bits give an update of 0, 8 bits a NaN, in their own element alone."""
    from paper_2608_15665_gb300 import firstorder as fo
    for bits in (32, 8):
        out = []
        for eps in (0.0, 1e-8):
            W = torch.ones(600, device=gpu)
            G = gradients(600, -20, 0, 9, gpu)
            G[77] = 1e25
            opt = fo.AdamW([W], [G], bits=bits)
            opt.step(1e-2, eps=eps, weight_decay=0.0)
            out.append(torch.isnan(W))
            assert (W[77] == 1.0) if bits == 32 else torch.isnan(W[77])
            opt.close()
        assert torch.equal(*out) and int(out[0].sum()) == (bits == 8)
