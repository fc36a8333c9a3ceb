"""Orthogonalised matrices whose squares leave fp32, in both directions: the result depends on
the matrix's direction alone (with eps = 0), whatever its scale.

Tolerances as in test_gpu_muon.py: 1.2e-5 of the result's norm for fp32 matrices and 4e-3 for bf16
ones.  Scaling by a power of two is exact; the entries that it makes subnormal lie 2^-100 below
the largest."""

import numpy as np
import pytest
import torch

from test_gpu_muon import TOL, TYPES, f64, gauss, ns, off

pytestmark = pytest.mark.gpu

# every kernel: rows in registers and in shared memory, one CTA and clusters, SM pairs
SHAPES = [(1, 1), (8, 900), (5120, 8), (24, 24), (16, 2000), (60, 60), (64, 1600), (128, 128),
          (100, 1000), (260, 300), (1030, 200)]
# 1e38 puts the Gaussians' largest entries near fp32's limit, 1e-38 most of them below its
# smallest normal number
SCALES = [3e37, 1e25, 1e20, 1e-14, 1e-20, 1e-30, 1e-38]


def scaled(m, n, dtype, dev, scale, seed=6):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, n, generator=g, dtype=torch.float64).clamp(-6, 6) * scale
    return x.to(torch.float32).to(TYPES[dtype]).to(dev)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n", SHAPES, ids=[f"{s[0]}x{s[1]}" for s in SHAPES])
def test_any_scale_gives_the_direction(lib, gpu, m, n, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    Gs = [scaled(m, n, dtype, gpu, s) for s in SCALES]
    out = fo.Orthogonalizer(Gs)(5, None, 0.0)
    torch.cuda.synchronize()
    for s, G, o in zip(SCALES, Gs, out):
        assert bool(torch.isfinite(G).all()) and float(G.abs().max()) > 0
        assert off(o, ns(f64(G), eps=0.0)) <= TOL[dtype], s


@pytest.mark.parametrize("m,n", [(8, 900), (60, 60), (100, 1000), (260, 300)])
def test_one_entry_far_above_the_rest(lib, gpu, m, n):
    """The rest keeps what the 2^-38 of the iterates leave of it: here nothing."""
    from paper_2608_15665_gb300 import firstorder as fo
    G = gauss(m, n, "f32", gpu, 3, scale=1e5)
    G[m // 2, n // 3] = -1e30
    out = fo.Orthogonalizer([G])(5, None, 0.0)[0]
    torch.cuda.synchronize()
    assert off(out, ns(f64(G), eps=0.0)) <= TOL["f32"]


@pytest.mark.parametrize("m,n", [(8, 900), (60, 60), (100, 1000), (260, 300)])
def test_an_eps_keeps_its_meaning(lib, gpu, m, n):
    """Beside a norm beyond fp32's squares eps is nothing; far above a tiny one it is all that is
    divided by, and the iterate, 2^-38 at most, is zero."""
    from paper_2608_15665_gb300 import firstorder as fo
    big, tiny = scaled(m, n, "f32", gpu, 1e25), scaled(m, n, "f32", gpu, 1e-30)
    out = fo.Orthogonalizer([big, tiny, torch.zeros_like(big)])(5, None, 1e-7)
    torch.cuda.synchronize()
    assert off(out[0], ns(f64(big), eps=0.0)) <= TOL["f32"]
    # an entry is below 1e-29 / 1e-7, and five steps take it up by 3.4445^5 = 485 at most
    assert float(out[1].abs().max()) <= 485 * 6e-30 / 1e-7
    assert float(out[2].abs().max()) == 0.0


@pytest.mark.parametrize("m,n", [(8, 900), (60, 60), (100, 1000), (260, 300)])
def test_muon_steps_from_momenta_beyond_the_squares(lib, gpu, m, n):
    from paper_2608_15665_gb300 import firstorder as fo
    for scale in (1e25, 1e-25):
        W = gauss(m, n, "f32", gpu, 5)
        G, M = scaled(m, n, "f32", gpu, scale, 7), scaled(m, n, "f32", gpu, 4 * scale, 8)
        before, mu = f64(W), float(np.float32(0.9))
        mom = mu * f64(M) + f64(G)
        want = before - 0.25 * ns(f64(G) + mu * mom, eps=0.0)
        opt = fo.Muon([W], [G], [M])
        opt.step(0.25, 0.9, True, 0.0, "none", eps=0.0)
        opt.sync()
        err = float((f64(W) - want).norm())
        assert err <= TOL["f32"] * 0.25 * float(ns(f64(G) + mu * mom, eps=0.0).norm()) \
            + 2 * 2.0 ** -24 * float(want.norm())
        assert float((f64(M) - mom).abs().max()) <= 2.0 ** -22 * float(mom.abs().max())
