"""AdamW's steps where the second moments leave fp32's normal numbers: gradients of 1e-22 to 1e-17,
and means that decay through 2^-126 to zero.

The moments are products and a sum, each rounded to fp32 with its subnormal numbers, so numpy's
fp32 arithmetic gives them bit for bit.  A code is floor(y + u), y the state in its block's steps and u
the random part: exact for normal codes; below them y is rounded once more, at 2^-20 of a step.  Roots
of v < 2^-102 may come out 2^-65 too small, which is nothing beside eps.  W's
update from those moments: the hardware's approximate division and root (2 ulp each), the
corrections rounded to fp32 (2 u each) and the products: 24 u of its magnitude, with u = 2^-24, and
2 u of W's, and half an ulp."""

import numpy as np
import pytest
import torch

from test_gpu_adamw import B1, B2, U, WD, f64, random_of, values

pytestmark = pytest.mark.gpu

f = np.float32


def moments(m, r, x, b2):
    """(m, v) of the next step in fp32 from m, r = sqrt(v) and the gradient."""
    m, r, x = (t.astype(f) for t in (m, r, x))
    return f(B1) * m + f(1.0 - B1) * x, f(b2) * (r * r) + f(1.0 - b2) * (x * x)


def codes_of(x, E, u):
    """(multiples of the blocks' powers of two, their codes' steps)"""
    y = np.abs(x) * 2.0 ** np.repeat(134.0 - np.maximum(E, 40), 256)[:x.size]
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(y, 1e-30))), -6) - 3)
    return y, np.floor(y / step + u) * step


def check_codes(codes, exps, x, E, u, positive):
    """codes of |x| (64 bits) in blocks of exponents E; roots below 2^-51 may be 2^-65 too small."""
    assert np.array_equal(exps.cpu().numpy(), E)
    c = f64(codes)
    assert np.all(np.isfinite(c)) and np.all(np.abs(c) <= 256)
    y, want = codes_of(x, E, u)
    exact = (y >= 2.0 ** -6) & ((np.abs(x) >= 2.0 ** -51) | (not positive))
    assert np.array_equal(np.abs(c)[exact], want[exact])
    less = np.abs(x) - (2.0 ** -65 * (np.abs(x) < 2.0 ** -51) if positive else 0.0)
    lo, hi = codes_of(np.maximum(less, 0.0), E, u - 2.0 ** -19)[1], codes_of(x, E, u + 2.0 ** -19)[1]
    if positive:
        assert np.all(c >= 0) and np.all((c > 0) == (x > 0))
        lo, hi = (np.where(x > 0, np.maximum(t, 2.0 ** -9), t) for t in (lo, hi))
    assert np.all((np.abs(c) >= lo) & (np.abs(c) <= hi))


def root_exponents(v):
    """of blocks: the biased exponents of the largest root, 63 where its v is subnormal"""
    pad = np.zeros(-(-v.size // 256) * 256, f)
    pad[:v.size] = v
    top = pad.reshape(-1, 256).max(1)
    k = np.maximum(np.frexp(top)[1] - 1, -126) >> 1
    return np.where(top > 0, np.where(top < f(2.0 ** -126), 63, k + 127), 0)


def check_w(got, W, m, v, t, lr, eps, b2=B2, wd=WD):
    hat = lr * m.astype(np.float64) / (1 - B1 ** t)
    step = hat / (np.sqrt(v.astype(np.float64) / (1 - b2 ** t)) + eps)
    want = (1 - lr * wd) * W - step
    lim = 2 * U * np.abs(W) + 24 * U * np.abs(step) + 1.01 * U * np.abs(want)
    assert np.all(np.abs(f64(got) - want) <= lim)


@pytest.mark.parametrize("scale", [1e-22, 1e-21, 1e-20, 1e-19, 3e-19, 1e-18, 3e-18, 1e-17, 1e-14])
def test_small_gradients_in_8_bits(lib, gpu, scale):
    from paper_2608_15665_gb300 import firstorder as fo
    n, lr, eps = 256 * 40 + 77, 1e-2, 1e-8
    g = torch.Generator().manual_seed(3)
    W = (torch.randn(n, generator=g) * 0.02).to(gpu)
    G = ((torch.rand(n, generator=g) + 0.5) * torch.randn(n, generator=g).sign() * scale).to(gpu)
    opt = fo.AdamW([W], [G], bits=8, seed=11)
    s = opt.states[0]
    for t in range(1, 5):
        before, x = f64(W), f64(G)
        m, r = values(s.m, s.m_exp, (n,)), values(s.v, s.v_exp, (n,))
        opt.step(lr, (B1, B2), eps, WD)
        torch.cuda.synchronize()
        m1, v1 = moments(m, r, x, B2)
        assert torch.isfinite(W).all()
        check_w(W, before, m1, v1, t, lr, eps)
        pad = np.zeros(41 * 256)
        pad[:n] = np.abs(m1)
        em = np.frexp(pad.reshape(-1, 256).max(1))[1] + 126
        u = random_of(11, 0, t, n)
        check_codes(s.m, s.m_exp, m1.astype(np.float64), np.maximum(em, 0), u, False)
        check_codes(s.v, s.v_exp, np.sqrt(v1).astype(np.float64), root_exponents(v1), u, True)
    opt.close()


def test_means_that_decay_to_nothing_in_8_bits(lib, gpu):
    """Zero gradients and b2 = 1/2: v halves a step, through the subnormal numbers to zero."""
    from paper_2608_15665_gb300 import firstorder as fo
    n, b2 = 512, 0.5
    g = torch.Generator().manual_seed(4)
    W = torch.randn(n, generator=g).to(gpu)
    G = torch.zeros(n, device=gpu)
    G[:256] = torch.randn(256, generator=g) * 2.0 ** -61
    G[256:] = torch.randn(256, generator=g) * 2.0 ** -68
    opt = fo.AdamW([W], [G], bits=8, seed=2)
    s = opt.states[0]
    for t in range(1, 61):
        before, x = f64(W), f64(G)
        m, r = values(s.m, s.m_exp, (n,)), values(s.v, s.v_exp, (n,))
        opt.step(1e-3, (B1, b2), 1e-8, 0.0)
        torch.cuda.synchronize()
        m1, v1 = moments(m, r, x, b2)
        check_w(W, before, m1, v1, t, 1e-3, 1e-8, b2, 0.0)
        check_codes(s.v, s.v_exp, np.sqrt(v1).astype(np.float64), root_exponents(v1),
                    random_of(2, 0, t, n), True)
        G.zero_()
    assert (s.v.float() == 0).all() and (s.v_exp == 0).all()
    opt.close()
