"""A pair's loss and its derivative from the 64-bit sums.

With one logit a row a label's log-probability is 0 exactly, so that D is the reference's part alone,
which 64 bits hold exactly; the formulas in 64 bits are then right to 2^-50.  Of what is returned, e =
exp(-|z|) is off by 5 u of itself (u = 2^-24: expf's 2 ulp and a rounding), log(1 + e) by 7 u (and log1pf's
ulp), e / (1 + e) by 7 u (and two roundings), and all by 2^-148 where they are subnormal; the rest is in 64
bits.  Results are rounded once: u."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("kind,smoothing,margin", [
    ("sigmoid", 0.0, 0.0), ("sigmoid", 0.1, 0.0), ("sigmoid", 0.3, 0.7), ("sigmoid", 0.0, -2.5),
    ("hinge", 0.0, 0.0), ("hinge", 0.0, 0.3), ("square", 0.0, 0.0)])
@pytest.mark.parametrize("beta", [0.1, 0.35, 3.0])
def test_losses_and_slopes_of_64_bit_sums(lib, gpu, kind, smoothing, margin, beta):
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

    both = far = 0.0                                   # what is made in fp32
    if kind == "sigmoid":
        both, far = np.log1p(np.exp(-np.abs(z))), np.exp(-np.logaddexp(0.0, np.abs(z)))

    def close(x, want, lim):
        lim = lim + U * np.abs(want) + 2.0 ** -148
        assert np.all(np.abs(x.double().cpu().numpy() - want) <= lim * (1 + 2.0 ** -20))
    # (64-bit roundings, here and there: of z, and of terms that cancel)
    rest = 2.0 ** -50 * (np.abs(z) + (1.0 if kind != "sigmoid" else 0.0) + (D * D + 0.25 / b ** 2) * (kind == "square"))
    err = 7 * U * both + rest * (np.minimum(1.0, both + a + (z < 0)) if kind == "sigmoid" else 1.0)
    close(got.losses, losses, err)
    # (their mean: of rounded losses, and rounded itself)
    close(got.loss, losses.mean(), err.mean() + U * np.abs(losses).mean())
    err = 7 * U * b * far + 2.0 ** -50 * (np.abs(slope) * (1 + np.abs(z)) + b * a + np.abs(D) * (kind == "square")
                                          + 0.5 / b * (kind == "square"))
    close(got.dlogp[:pairs], slope / pairs, err / pairs)
    assert torch.equal(got.dlogp[pairs:], -got.dlogp[:pairs])


def test_pairs_without_end(lib, gpu):
    """References of infinity: the losses' limits, as for any far pair."""
    from paper_2608_15665_gb300 import firstorder as fo
    inf = float("inf")
    ref = torch.tensor([inf, -inf, 0.0, 0.0, 0.0, 0.0], device=gpu)       # D = -inf, inf, 0
    args = (torch.zeros(6, 1, device=gpu), torch.zeros(6, dtype=torch.int64, device=gpu),
            torch.arange(7, device=gpu), ref)
    got = fo.preference_loss(*args, 0.5)
    assert got.losses[:2].tolist() == [inf, 0.0] and float(got.losses[2]) == pytest.approx(np.log(2.0))
    assert (3 * got.dlogp[:3]).tolist() == pytest.approx([-0.5, 0.0, -0.25])
    got = fo.preference_loss(*args, 0.5, "sigmoid", 0.25)
    assert got.losses[:2].tolist() == [inf, inf]
    assert (3 * got.dlogp[:3]).tolist() == pytest.approx([-0.375, 0.125, -0.125])
    got = fo.preference_loss(*args, 0.5, "hinge")
    assert got.losses.tolist() == [inf, 0.0, 1.0] and (3 * got.dlogp[:3]).tolist() == pytest.approx([-0.5, 0.0, -0.5])
