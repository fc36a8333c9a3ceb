"""Newton-Schulz orthogonalisation and the Muon step against their definition in 64 bits.

Tolerances, in the Frobenius norm relative to the result's, derived before the first run.
fp32 matrices: iterates and products of ~2^-22, about ten roundings a step; a step's map has
slopes up to 3.44 on small singular values and about 1 on those near 1, and rounding noise,
spread over all directions, grows no faster than the result's own norm, which starts at 1 and
ends near sqrt(rank): 10 x 5 x 2^-22 = 1.2e-5.  bf16 matrices: rounding the result gives
2^-9 / sqrt(3) x ~1.5 = 1.7e-3; the single fp16 factors of the last two steps 2^-12 x
(|b| s + 2 |c| s^2 ~ 8) / sqrt(3) a product = 1.1e-3 each: sqrt(1.7^2 + 4 x 1.1^2) 1e-3 =
2.8e-3, and 4e-3 with a margin for the few directions of the smallest matrices."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
TOL = {"bf16": 4e-3, "f32": 1.2e-5}
QUINTIC = (3.4445, -4.7750, 2.0315)


def f64(t):
    return t.detach().float().cpu().double()


def ns(U, steps=5, coeffs=None, eps=1e-7):
    """The definition in 64 bits, by the singular values."""
    U = U.double()
    norm = float(torch.linalg.vector_norm(U)) + eps
    if norm == 0:
        return U
    left, s, right = torch.linalg.svd(U / norm, full_matrices=False)
    for k in range(steps):
        a, b, c = [float(np.float32(v)) for v in (coeffs[k] if coeffs else QUINTIC)]
        s = a * s + b * s ** 3 + c * s ** 5
    return (left * s) @ right


def gauss(m, n, dtype, dev, seed, pad=0, spread=0.0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, n, generator=g) * torch.exp(spread * torch.randn(1, n, generator=g)) * scale
    buf = torch.full((m, n + pad), float("nan"))
    buf[:, :n] = x
    return buf.to(TYPES[dtype]).to(dev)[:, :n]


def off(got, want):
    d = f64(got) - want
    return float(torch.linalg.vector_norm(d) / torch.linalg.vector_norm(want))


def check(got, want, dtype):
    assert bool(torch.isfinite(got).all())
    assert off(got, want) <= TOL[dtype]
    rms = float(torch.linalg.vector_norm(want)) / want.numel() ** 0.5
    far = (f64(got) - want).abs() / want.abs().clamp_min(rms)
    assert float(far.max()) <= 12 * TOL[dtype]


SHAPES = [(1, 1, 0), (1, 7, 0), (5, 1, 0), (4, 4, 0), (8, 8, 3), (16, 16, 0), (17, 33, 0),
          (32, 32, 0), (48, 64, 0), (64, 64, 1), (100, 100, 0), (128, 128, 0), (128, 96, 0),
          (129, 130, 0), (8, 5120, 0), (5120, 8, 0), (16, 2000, 5), (1500, 32, 0), (64, 1408, 0),
          (200, 1000, 0), (1000, 200, 7), (256, 256, 0), (257, 511, 1), (512, 257, 0), (640, 640, 0),
          (333, 1001, 0), (1024, 520, 8), (768, 1536, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,pad", SHAPES, ids=[f"{s[0]}x{s[1]}" for s in SHAPES])
def test_orthogonalize_matches_the_definition(lib, gpu, m, n, pad, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    G = gauss(m, n, dtype, gpu, 3, pad, spread=0.5)
    out = gauss(m, n, dtype, gpu, 4, pad)
    op = fo.Orthogonalizer([G], [out])
    op()
    op.sync()
    check(out, ns(f64(G)), dtype)
    if pad:                                              # the padding is not written
        assert bool(torch.isnan(torch.as_strided(out, (m, pad), out.stride(), n)).all())
    first = out.clone()
    out.fill_(float("nan"))                              # the old contents are not read
    op()
    op.close()
    assert torch.equal(first, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,pad", [(48, 7680, 0), (7681, 33, 3), (130, 8192, 0), (200, 6001, 1),
                                     (4097, 257, 0)])
def test_few_rows_of_great_length(lib, gpu, m, n, pad, dtype):
    """Gram's K in several parts, whose sums are added in one order whoever finishes last."""
    from paper_2608_15665_gb300 import firstorder as fo
    G = gauss(m, n, dtype, gpu, 13, pad, spread=0.5)
    op = fo.Orthogonalizer([G, G])
    first = [o.clone() for o in op()]
    for _ in range(8):
        again = op()
    op.sync()
    check(first[0], ns(f64(G)), dtype)
    for t in (first[1], again[0], again[1]):
        assert torch.equal(first[0], t)
    op.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,pad", [(7, 4999, 1), (3, 641, 0), (8, 5136, 0), (4801, 6, 2), (2, 130, 0),
                                     (9, 5120, 0), (16, 641, 3)])
def test_at_most_sixteen_rows(lib, gpu, m, n, pad, dtype):
    """X in registers or in shared memory, clusters whose last CTA has few columns or none."""
    from paper_2608_15665_gb300 import firstorder as fo
    G = gauss(m, n, dtype, gpu, 17, pad, spread=0.5)
    W = gauss(m, n, dtype, gpu, 18, pad)
    op = fo.Orthogonalizer([G])
    first = op()[0].clone()
    check(first, ns(f64(G)), dtype)
    assert torch.equal(first, op()[0])
    op.close()
    before, mu = f64(W), fo.Muon([W], [G])
    mu.step(0.25, 0.0, False, 0.0, "none")
    mu.sync()
    want = before - 0.25 * ns(f64(G))
    ulp = 2.0 ** -9 if dtype == "bf16" else 2.0 ** -24
    err = float((f64(W) - want).norm())
    assert err <= TOL[dtype] * 0.25 * float(ns(f64(G)).norm()) + 2 * ulp * float(want.norm())
    mu.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ill_conditioned_matrices(lib, gpu, dtype):
    """Singular values falling as 1 / k, and a few strong directions over a noise floor: the
    small ones end far from 1, and are those that rounding noise meets first."""
    from paper_2608_15665_gb300 import firstorder as fo
    g = torch.Generator().manual_seed(8)
    cases = []
    for m, n in ((96, 96), (300, 500), (512, 512)):
        q = torch.linalg.qr(torch.randn(m, min(m, n), generator=g))[0]
        w = torch.linalg.qr(torch.randn(n, min(m, n), generator=g))[0]
        cases.append((q / torch.arange(1, min(m, n) + 1)) @ w.t())
        cases.append(torch.randn(m, 8, generator=g) @ torch.randn(8, n, generator=g)
                     + 0.05 * torch.randn(m, n, generator=g))
    Gs = [c.to(TYPES[dtype]).to(gpu) for c in cases]
    out = fo.Orthogonalizer(Gs)()
    torch.cuda.synchronize()
    for G, o in zip(Gs, out):
        # the noise's slope on the smallest values is 3.44^5 = 485, theirs the same: their own
        # digits are lost where the largest value's 2^-22 reaches them
        assert off(o, ns(f64(G))) <= (TOL[dtype] if dtype == "bf16" else 5 * TOL[dtype])


@pytest.mark.parametrize("steps,coeffs", [
    (1, None), (3, None), (10, None), (6, [(1.5, -0.5, 0.0)] * 6),
    (3, [(3.4, -4.7, 2.0), (3.0, -3.2, 1.2), (1.875, -1.25, 0.375)]),
])
@pytest.mark.parametrize("m,n", [(48, 40), (300, 260)])
def test_steps_and_coefficients(lib, gpu, m, n, steps, coeffs):
    from paper_2608_15665_gb300 import firstorder as fo
    G = gauss(m, n, "f32", gpu, 5)
    out = fo.Orthogonalizer([G])(steps, coeffs, 1e-7)[0]
    torch.cuda.synchronize()
    want = ns(f64(G), steps, coeffs)
    assert off(out, want) <= TOL["f32"] * max(2, steps) / 2


def test_coefficients_that_leave_the_range_are_refused(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    op = fo.Orthogonalizer([gauss(8, 8, "f32", gpu, 5)])
    before = op.outputs[0].clone()
    n = lib.zo_muon_launches(op.ctx)
    # the second: 1 -> 2.2 -> 6.2 -> 4200
    for steps, coeffs, eps in ((5, [(30.0, 5.0, 9.0)] * 5, 1e-7),
                               (4, [(8.2, -22.0, 16.0), (4.0, -2.9, 0.55), (3.9, -2.8, 0.53),
                                    (3.3, -2.4, 0.46)], 1e-7), (0, None, 1e-7),
                               (33, None, 1e-7), (1, [(float("nan"), 0, 0)], 1e-7),
                               (1, [(1e20, 0, 0)], 1e-7), (5, None, -1.0),
                               (5, None, float("inf"))):
        with pytest.raises(lib.ZoError) as e:
            op(steps, coeffs, eps)
        assert e.value.status == lib.ZO_ERR_INVALID_ARG
    mu = fo.Muon([gauss(8, 8, "f32", gpu, 5)])
    for kw in (dict(lr=float("nan")), dict(lr=0.1, momentum=1.0), dict(lr=0.1, momentum=-0.1),
               dict(lr=0.1, weight_decay=float("inf")), dict(lr=0.1, eps=-1.0)):
        with pytest.raises(lib.ZoError):
            mu.step(**kw)
    assert lib.zo_muon_launches(op.ctx) == n and lib.zo_muon_launches(mu.ctx) == 0
    torch.cuda.synchronize()
    assert torch.equal(before.nan_to_num(0.5), op.outputs[0].nan_to_num(0.5))


def mixed(dev):
    """Matrices of many shapes and both types, in an order that mixes them."""
    shapes = [(32, 32), (300, 200), (8, 700), (64, 64), (1, 5), (700, 8), (520, 640), (128, 128),
              (20, 20), (200, 300), (96, 1000), (4, 4), (513, 260)]
    return [gauss(m, n, "bf16" if k % 2 else "f32", dev, 20 + k, pad=k % 3)
            for k, (m, n) in enumerate(shapes)]


def test_a_set_gives_each_matrix_its_own_bits(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    Gs = mixed(gpu)
    whole = fo.Orthogonalizer(Gs)()
    alone = [fo.Orthogonalizer([G])()[0] for G in Gs]
    torch.cuda.synchronize()
    for G, a, b in zip(Gs, whole, alone):
        assert torch.equal(a, b)
        check(a, ns(f64(G)), "bf16" if G.dtype == torch.bfloat16 else "f32")


def test_several_groups_share_the_buffers(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    Gs = [gauss(1100, 60000, "bf16", gpu, 40 + k) for k in range(4)]   # > 1 GiB of iterates
    Gs.insert(2, gauss(30, 40, "bf16", gpu, 50))
    whole = fo.Orthogonalizer(Gs)()
    torch.cuda.synchronize()
    for G, a in zip(Gs, whole):
        assert torch.equal(fo.Orthogonalizer([G])()[0], a)
    o = whole[3].float()
    spread = (o @ o.t()).diagonal()                      # near-orthonormal rows
    assert 0.4 < float(spread.min()) and float(spread.max()) < 1.5


@pytest.mark.parametrize("m,n", [(24, 24), (8, 900), (60, 60), (128, 128), (260, 300)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zero_tiny_huge_and_non_finite_matrices(lib, gpu, m, n, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    base = gauss(m, n, dtype, gpu, 6)
    nan, inf = base.clone(), base.clone()
    nan[m // 2, n // 3] = float("nan")
    inf[m - 1, 0] = float("inf")
    Gs = [torch.zeros_like(base), base * 1e-3, base * 1e12, nan, inf, base]
    out = fo.Orthogonalizer(Gs)(5, None, 0.0)
    torch.cuda.synchronize()
    assert float(out[0].abs().max()) == 0.0
    for k in (1, 2, 5):
        assert off(out[k], ns(f64(Gs[k]), eps=0.0)) <= TOL[dtype]
    assert bool(torch.isnan(out[3]).all()) and bool(torch.isnan(out[4]).all())


def muon_reference(W, G, M, lr, momentum, nesterov, wd, adjust):
    m, n = W.shape
    if M is not None:
        M = momentum * M + G
        U = G + momentum * M if nesterov else M
    else:
        U = G
    s = {"none": 1.0, "aspect": max(1.0, m / n) ** 0.5, "rms": 0.2 * max(m, n) ** 0.5}[adjust]
    return (1 - lr * wd) * W - lr * s * ns(U), M


@pytest.mark.parametrize("dtype,gdtype", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"),
                                          ("f32", "bf16")])
@pytest.mark.parametrize("nesterov,wd,adjust", [(True, 0.1, "aspect"), (False, 0.0, "rms"),
                                                (True, 0.0, "none")])
def test_muon_steps_match_the_definition(lib, gpu, dtype, gdtype, nesterov, wd, adjust):
    from paper_2608_15665_gb300 import firstorder as fo
    shapes = [(40, 40), (8, 600), (600, 16), (300, 270), (130, 400), (1, 9)]
    lr, mu = 0.25, 0.9                       # binary fractions of lr keep keep = 1 - lr wd exact
    W = [gauss(m, n, dtype, gpu, 60 + k, pad=k % 2) for k, (m, n) in enumerate(shapes)]
    G = [gauss(m, n, gdtype, gpu, 70 + k, pad=(k + 1) % 3) for k, (m, n) in enumerate(shapes)]
    M = [gauss(m, n, "f32", gpu, 80 + k) for k, (m, n) in enumerate(shapes)]
    M[2] = None                              # one matrix without momentum
    opt = fo.Muon(W, G, M)
    for step in range(2):
        before = [(f64(w), f64(g), None if x is None else f64(x)) for w, g, x in zip(W, G, M)]
        opt.step(lr, mu, nesterov, wd, adjust)
        opt.sync()
        for k, (w, g, x) in enumerate(before):
            lr32, mu32, wd32 = (float(np.float32(v)) for v in (lr, mu, wd))
            want, mom = muon_reference(w, g, x, lr32, mu32, nesterov, wd32, adjust)
            o = (want - (1 - lr32 * wd32) * w).norm()    # the update's size
            err = (f64(W[k]) - want).norm()
            ulp = 2.0 ** -9 if dtype == "bf16" else 2.0 ** -24
            assert float(err) <= TOL[dtype] * float(o) + 2 * ulp * float(want.norm())
            if x is not None:
                assert float((f64(M[k]) - mom).abs().max()) <= 2.0 ** -22 * float(mom.abs().max())
        for k, g in enumerate(G):            # the next step's gradient, in the same buffers
            g.copy_(gauss(*shapes[k], gdtype, gpu, 90 + 10 * step + k))


def test_back_to_back_steps_and_a_stream_of_ones_own(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo

    def train(stream):
        W = [gauss(m, n, "bf16", gpu, 5 + k) for k, (m, n) in enumerate([(64, 64), (300, 520), (8, 900)])]
        G = [gauss(*w.shape, "bf16", gpu, 30 + k) for k, w in enumerate(W)]
        torch.cuda.synchronize()
        opt = fo.Muon(W, G, stream=stream)
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            for t in range(5):
                opt.step(0.05, 0.9)
                for g in G:
                    g.mul_(-0.75)            # on the same stream, between the steps
        opt.sync()
        torch.cuda.synchronize()
        return W + opt.momenta
    for a, b in zip(train(None), train(torch.cuda.Stream())):
        assert torch.equal(a, b)


def test_a_captured_step_replays_on_new_contents(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    s = torch.cuda.Stream()
    Gs = mixed(gpu)
    W = [torch.zeros_like(G) for G in Gs]
    with torch.cuda.stream(s):
        opt = fo.Muon(W, Gs, stream=s)
        opt.step(0.5, 0.9)                   # set-up that a first launch does
        opt.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            opt.step(0.5, 0.9)
        for t in list(W) + opt.momenta:
            t.zero_()
        for t in range(3):
            graph.replay()
            for g in Gs:
                g.mul_(0.5)
        s.synchronize()
    want_g = mixed(gpu)
    want_w = [torch.zeros_like(G) for G in want_g]
    live = fo.Muon(want_w, want_g)
    for t in range(3):
        live.step(0.5, 0.9)
        for g in want_g:
            g.mul_(0.5)
    torch.cuda.synchronize()
    for a, b in zip(W + opt.momenta, want_w + live.momenta):
        assert torch.equal(a, b)


def test_no_device_memory_is_allocated_by_calls(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    opt = fo.Muon([gauss(300, 400, "bf16", gpu, 1), gauss(16, 16, "f32", gpu, 2)])
    opt.step(0.1)
    torch.cuda.synchronize()
    free0 = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        opt.step(0.1)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free0
