"""A pair's loss and its derivative from the 64-bit sums: rounded once, at the end.

With one logit a row a label's log-probability is 0 exactly, so that D is the reference's part alone,
which 64 bits hold exactly; the formulas in 64 bits are then right to 2^-50, and what is returned is off
by half an ulp (2^-24 of it) at most, or by half of the smallest subnormal number."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("kind,smoothing,margin", [
    ("sigmoid", 0.0, 0.0), ("sigmoid", 0.1, 0.0), ("sigmoid", 0.3, 0.7), ("sigmoid", 0.0, -2.5),
    ("hinge", 0.0, 0.0), ("hinge", 0.0, 0.3), ("square", 0.0, 0.0)])
@pytest.mark.parametrize("beta", [0.1, 0.35, 3.0])
def test_losses_and_slopes_are_rounded_once(lib, gpu, kind, smoothing, margin, beta):
    from paper_2608_15665_gb300 import firstorder as fo
    g = torch.Generator().manual_seed(5)
    pairs = 3000
    size = 10.0 ** (torch.rand(pairs, generator=g) * 6 - 4)
    chosen = torch.randn(pairs, generator=g).sign() * size
    rejected = torch.randn(pairs, generator=g) * 10.0
    ref = torch.cat([chosen, rejected])
    rows = 2 * pairs
    got = fo.preference_loss(torch.randn(rows, 1, generator=g).to(gpu),
                             torch.zeros(rows, dtype=torch.int64, device=gpu),
                             torch.arange(rows + 1, device=gpu), ref.to(gpu), beta, kind, smoothing, margin)
    assert (got.logps == 0).all()
    D = -(ref[:pairs].double().numpy() - ref[pairs:].double().numpy())
    b, a, shift = (float(np.float32(t)) for t in (beta, smoothing, margin))
    z = b * D - shift
    if kind == "square":
        losses, slope = (D - 0.5 / b) ** 2, 2 * (D - 0.5 / b)
    elif kind == "hinge":
        losses, slope = np.maximum(0.0, 1.0 - z), np.where(z < 1.0, -b, 0.0)
    else:
        losses = (1 - a) * np.logaddexp(0.0, -z) + a * np.logaddexp(0.0, z)
        slope = b * (a * np.exp(-np.logaddexp(0.0, -z)) - (1 - a) * np.exp(-np.logaddexp(0.0, z)))

    def once(x, want, terms):
        lim = U * (1 + 2.0 ** -20) * np.abs(want) + 2.0 ** -150 + 2.0 ** -50 * terms
        assert np.all(np.abs(x.double().cpu().numpy() - want) <= lim)
    # (64-bit roundings of terms that cancel: of z and 1, of the slope's two parts)
    terms = np.abs(z) + 1.0 + (D * D + 0.25 / b ** 2) * (kind == "square")
    small = 0.0 if kind == "sigmoid" and a == 0.0 else terms
    once(got.losses, losses, small + np.abs(losses) * (1 + np.abs(z)))
    # (their mean: of rounded losses, and rounded itself)
    assert abs(float(got.loss) - losses.mean()) <= 2 * U * (1 + 2.0 ** -20) * np.abs(losses).mean() + 2.0 ** -50 * terms.mean()
    grow = np.abs(slope) * (1 + np.abs(z)) + (b * a if kind == "sigmoid" else 0.0) + np.abs(D) * (kind == "square")
    once(got.dlogp[:pairs], slope / pairs, grow / pairs)
    assert torch.equal(got.dlogp[pairs:], -got.dlogp[:pairs])
