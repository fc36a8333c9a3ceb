"""The error of fp32-grade orthogonalisations of few rows against that of an fp32 evaluation.

A step of the kernels stores X, A and B as pairs of fp16, 1.6 times as coarse (in the mean square)
as fp32, and their products lose 2^-24 of their terms at most; a step in fp32 stores the same three
and rounds every sum of its products besides, over 4 to 8000 terms.  So the kernels' mean error over
a set may be a fifth above fp32's where sums are short, and no more; a set is large enough for its
mean to vary by a few percent."""

import pytest
import torch

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315


def _plain(U):
    tall = U.shape[1] > U.shape[2]
    X = U.transpose(1, 2) if tall else U
    X = X / (X.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    for _ in range(5):
        M = torch.bmm(X, X.transpose(1, 2))
        X = A * X + torch.bmm(B * M + C * torch.bmm(M, M), X)
    return X.transpose(1, 2) if tall else X


def _exact(U):
    U = U.double()
    U = U / (U.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    left, s, right = torch.linalg.svd(U, full_matrices=False)
    for _ in range(5):
        s = s * (A + s * s * (B + C * s * s))
    return (left * s[:, None, :]) @ right


@pytest.mark.parametrize("m,n,count", [
    (4, 4, 896), (8, 8, 896), (16, 16, 448), (64, 64, 112), (8, 256, 80), (8, 5120, 40), (5120, 8, 40),
    (4, 8000, 40), (8, 8000, 40), (16, 300, 80), (16, 2048, 40), (12, 5000, 20), (48, 96, 60),
    (64, 256, 30)])
def test_a_set_is_as_near_as_fp32_takes_it(lib, gpu, m, n, count):
    from paper_2608_15665_gb300 import firstorder as fo
    g = torch.Generator().manual_seed(m * 10007 + n)
    G = torch.randn(count, m, n, generator=g).to(gpu)
    got = torch.stack(fo.Orthogonalizer(list(G.unbind(0)))())
    want = _exact(G)

    def off(x):
        return ((x.double() - want).square().sum((1, 2)) / want.square().sum((1, 2))).sqrt()
    assert float(off(got).mean()) <= 1.2 * float(off(_plain(G)).mean())
