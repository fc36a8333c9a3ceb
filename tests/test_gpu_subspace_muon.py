"""zo_step with ZO_OPT_MUON: the orthogonalised first moment as the subspace direction.

The direction's error is the orthogonalisation's (fp32 grade, 1.2e-5 of its Frobenius norm:
test_gpu_muon.py); U and V are column-orthonormal, so it reaches W with the same norm.  The
moment's own error, relative 1e-5 of its terms as for Adam's, passes through the quintic's
steps with slopes of about 1 on the values that have reached 1, and up to 3.44^5 = 485 on
those that have not, for at most sqrt(r) 1e-6 = 1e-5 of the direction's norm at the fp32
roundings (2^-24) a moment of few terms has: 3e-5 together, and with the pass's own 2^-21 and
the weights' rounding (half an ulp of every element) the bound below."""

import numpy as np
import pytest
import torch

from gpu_util import f32, make_weight, snapshot
from oracle import subzero
from parity import assert_rel_scaled, gabs

pytestmark = pytest.mark.gpu

QUINTIC = tuple(float(np.float32(v)) for v in (3.4445, -4.7750, 2.0315))


def ns(M, eps):
    left, s, right = np.linalg.svd(M / (np.linalg.norm(M) + eps))
    a, b, c = QUINTIC
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    return (left * s) @ right


CASES = [("f32", 4, [(48, 60), (8, 200)]), ("f32", 8, [(64, 64)]), ("bf16", 16, [(96, 128), (40, 64)]),
         ("f32", 16, [(100, 36)]), ("bf16", 32, [(256, 320), (160, 96)]), ("bf16", 64, [(200, 264)]),
         ("f32", 64, [(130, 70)]), ("bf16", 128, [(300, 136), (256, 256)]), ("f32", 128, [(140, 129)])]


@pytest.mark.parametrize("dtype,r,shapes", CASES, ids=[f"{c[0]}-r{c[1]}" for c in CASES])
def test_steps_match_the_definition(lib, gpu, dtype, r, shapes):
    from paper_2608_15665_gb300 import binding as zb
    from paper_2608_15665_gb300.schedule import SubZeroPlus
    seed, q, eps, lr, beta1 = 77, 3, 1e-2, 0.5, 0.75
    # (a context wants row strides of 16 bytes)
    z = SubZeroPlus([make_weight(m, n, dtype, 5 + k, gpu, ldw=(n + 7) // 8 * 8)
                     for k, (m, n) in enumerate(shapes)], r, q, seed)
    z.init_subspace(0)
    for Vm in z.Vm:
        Vm.fill_(7.0)
    gamma = torch.empty(len(shapes), device=gpu)
    for t in range(2):
        before = snapshot(z)
        rho = np.asarray([1.5, -0.75, 0.25 + t], np.float32)
        restore = (1, -1.0) if t == 0 else (-1, 0.0)
        z.step(t, 1, rho, "direct", eps, lr, beta1, 0.0, 1e-8, restore[0], restore[1],
               optimizer=zb.ZO_OPT_MUON, gamma_out=gamma)
        z.sync()
        after = snapshot(z)
        for i in range(len(shapes)):
            G = subzero.grad_G(seed, i, t, r, rho.astype(np.float64))
            M = beta1 * before["M"][i] + (1 - beta1) * G
            scale = beta1 * np.abs(before["M"][i]) + (1 - beta1) * gabs(seed, i, t, r, rho)
            assert_rel_scaled(after["M"][i], M, scale, f"M {i}")
            assert np.all(after["Vm"][i] == 7.0)
            assert float(gamma[i]) == pytest.approx(np.linalg.norm(G), rel=1e-5)
            # from the moment that the GPU holds: what is tested is the direction
            D = ns(after["M"][i], f32(1e-8))
            terms = [restore] if restore[0] >= 0 else []
            C = subzero.step_coeff(D, f32(lr), f32(eps), terms, seed, i, t, r)
            want = before["W"][i] + before["U"][i] @ C @ before["V"][i].T
            ulp = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
            half = 0.5 * ulp * np.linalg.norm(np.abs(want) + np.abs(before["W"][i]))
            err = np.linalg.norm(after["W"][i] - want)
            assert err <= (3e-5 + 2.0 ** -20) * np.linalg.norm(C) + half, (i, err)
            # and W moved by the direction, not by a fraction of it
            assert np.linalg.norm(after["W"][i] - before["W"][i]) >= 0.9 * np.linalg.norm(C) - half
    z.close()


@pytest.mark.parametrize("dtype,r", [("f32", 8), ("bf16", 32), ("bf16", 128)])
def test_a_zero_moment_leaves_the_weights_and_repeats_agree(lib, gpu, dtype, r):
    from paper_2608_15665_gb300 import binding as zb
    from paper_2608_15665_gb300.schedule import SubZeroPlus
    W0 = make_weight(200, 168, dtype, 3, gpu)
    first = None
    for _ in range(2):
        z = SubZeroPlus([W0.clone()], r, 2, 5)
        z.init_subspace(0)
        z.step(0, 1, np.zeros(2, np.float32), "direct", 1e-3, 0.1, 0.9, 0.0, 1e-8, -1, 0.0,
               optimizer=zb.ZO_OPT_MUON)
        z.sync()
        assert torch.equal(z.weights[0], W0)               # NS(0) = 0
        z.step(1, 2, np.ones(2, np.float32), "direct", 1e-3, 0.1, 0.9, 0.0, 1e-8, -1, 0.0,
               optimizer=zb.ZO_OPT_MUON)
        z.sync()
        assert not torch.equal(z.weights[0], W0)
        first = z.weights[0] if first is None else first
        assert torch.equal(first, z.weights[0])


def test_it_is_the_full_matrices_orthogonalisation(lib, gpu):
    """U NS(M) V^T = NS(U M V^T): the subspace step moves W as zo_muon_step moves it on the
    full gradient.  The full matrix has min(m, n) - r zero singular values, whose rounding
    noise of 2^-22 grows by 485 at most: 1.2e-4, on a result of norm sqrt(r) = 4."""
    from paper_2608_15665_gb300 import binding as zb
    from paper_2608_15665_gb300 import firstorder as fo
    from paper_2608_15665_gb300.schedule import SubZeroPlus
    r = 16
    W = torch.zeros(160, 96, device=gpu)
    z = SubZeroPlus([W], r, 2, 9)
    z.init_subspace(0)
    z.step(0, 1, np.asarray([1.0, -0.5], np.float32), "direct", 1e-3, 1.0, 0.0, 0.0, 0.0, -1, 0.0,
           optimizer=zb.ZO_OPT_MUON)
    z.sync()
    full = z.U[0].double() @ z.M[0].double() @ z.V[0].double().t()
    O = fo.Orthogonalizer([full.float()])(5, None, 0.0)[0]
    torch.cuda.synchronize()
    assert float((O + W).norm() / O.norm()) <= 1.2e-4


def test_bad_scalars_are_refused(lib, gpu):
    from paper_2608_15665_gb300 import binding as zb
    from paper_2608_15665_gb300.schedule import SubZeroPlus
    W = make_weight(64, 64, "f32", 3, gpu)
    z = SubZeroPlus([W], 8, 2, 5)
    z.init_subspace(0)
    z.sync()
    before, n = W.clone(), zb.zo_kernel_launches(z.ctx)
    for beta1, eps in ((1.0, 1e-8), (-0.1, 1e-8), (0.9, -1.0), (0.9, float("inf"))):
        with pytest.raises(zb.ZoError) as e:
            z.step(0, 1, np.ones(2, np.float32), "direct", 1e-3, 0.1, beta1, 0.0, eps, -1, 0.0,
                   optimizer=zb.ZO_OPT_MUON)
        assert e.value.status == zb.ZO_ERR_INVALID_ARG
    with pytest.raises(zb.ZoError):
        z.step(0, 1, np.ones(2, np.float32), "direct", 1e-3, 0.1, 0.9, 0.0, 1e-8, -1, 0.0, optimizer=3)
    torch.cuda.synchronize()
    assert torch.equal(before, W) and zb.zo_kernel_launches(z.ctx) == n
