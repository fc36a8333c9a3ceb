"""bf16 matrices whose products are asked for in fp32 grade: what is left of the error is the
result's own rounding.

The rounding alone puts a result 2^-9 / sqrt(3) of its elements away, about 1.7e-3 of its norm
over a binade's spread; products of fp32 grade add 1.2e-5 at most (test_gpu_muon.py), in
quadrature nothing, and elements that lie within it of a rounding boundary, fewer than 1.2e-5 /
2^-8 of them at twice the error: 0.6%.  So 1.02 of the rounding's own error is asked for."""

import pytest
import torch

from test_gpu_muon import TOL, f64, gauss, ns, off

pytestmark = pytest.mark.gpu

SHAPES = [(129, 130), (256, 300), (1000, 200), (300, 1100), (640, 640)]


@pytest.mark.parametrize("m,n", SHAPES, ids=[f"{s[0]}x{s[1]}" for s in SHAPES])
def test_only_the_results_rounding_is_left(lib, gpu, m, n):
    from paper_2608_15665_gb300 import firstorder as fo
    G = gauss(m, n, "bf16", gpu, 3, spread=0.5)
    want = ns(f64(G))
    alone = off(want.to(torch.bfloat16), want)
    assert off(fo.Orthogonalizer([G], precise=True)()[0], want) <= 1.02 * alone
    # W = 0 and no momentum: the step's result is rounded once too
    W = torch.zeros_like(G)
    opt = fo.Muon([W], [G], precise=True)
    opt.step(1.0, momentum=0.0, nesterov=False, adjust="none")
    opt.sync()
    assert off(W, -want) <= 1.02 * alone
    # without it, within the tolerance that is stated for single factors
    assert off(fo.Orthogonalizer([G])()[0], want) <= TOL["bf16"]


def test_matrices_that_have_it_anyway_are_unchanged(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    Gs = [gauss(*s, t, gpu, 9) for s, t in (((300, 260), "f32"), ((128, 400), "bf16"), ((20, 20), "bf16"))]
    plain, asked = fo.Orthogonalizer(Gs)(), fo.Orthogonalizer(Gs, precise=True)()
    torch.cuda.synchronize()
    for a, b in zip(plain, asked):
        assert torch.equal(a, b)
