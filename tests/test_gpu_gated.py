"""The gated linear block on the GPU against its formulas in 64 bits, on the same inputs.

Tolerances, per element, derived before the first run.  A product of K bf16 pairs is exact in each
pair; sixteen are added to the fp32 accumulator at a time, which rounds towards zero: at most
(K / 16 + 16) 2^-23 of the sum of magnitudes.  act comes from s = 1 / (1 + exp(-y)), off by
(32 + |y|) 2^-22 of itself (the exponential's argument and the approximate functions).  H is off by its
factors' errors (|act'| <= 1.13), dG = dH U s (1 + g y' (1 - s)) by the magnitudes of its terms.  dG
and dU are rounded to bf16 (half a step, 2^-9): the reference rounds them too, and where their errors reach
over a rounding's border the step between the two sides counts; up to 128 tokens they are sums of two
bf16, within 2^-17.  Every result is rounded once:
2^-8 of it at most."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

C = 2 * np.sqrt(2 / np.pi)
BF = torch.bfloat16


def make(rows, cols, dev, seed, scale=1.0, pad=0):
    """A bf16 matrix in rows `pad` elements apart, NaN between them."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((rows, cols + pad), float("nan"))
    buf[:, :cols] = torch.randn(rows, cols, generator=g) * scale
    return buf.to(BF).to(dev)[:, :cols]


def inputs(T, D, F, dev, pad=0):
    s = 1.2 / np.sqrt(D)
    return make(T, D, dev, 1, 1.0, pad), make(F, D, dev, 2, s, pad), make(F, D, dev, 3, s, pad)


def gate(g, act):
    """(s, y, y')"""
    if act == "silu":
        y, y1 = g, torch.ones_like(g)
    else:
        y, y1 = C * (g + 0.044715 * g ** 3), C * (1 + 3 * 0.044715 * g * g)
    return torch.sigmoid(y), y, y1


def bf16(x):
    return x.to(torch.float32).to(BF).double()


def accumulation(K):
    return (K / 16 + 16) * 2.0 ** -23


def close(got, want, lim):
    off = (got.double() - want).abs() - lim - 2.0 ** -8 * want.abs() - 2.0 ** -133
    assert float(off.max()) <= 0, float(off.max())


def check_forward(out, x, wg, wu, act):
    X, Wg, Wu = x.double(), wg.double(), wu.double()
    G, U = X @ Wg.t(), X @ Wu.t()
    a = accumulation(X.shape[1])
    eg, eu = a * (X.abs() @ Wg.abs().t()), a * (X.abs() @ Wu.abs().t())
    s, y, _ = gate(G, act)
    H = G * s * U
    close(out.h, H, 1.13 * U.abs() * eg + (G * s).abs() * eu + 1.13 * eg * eu
          + H.abs() * (34 + y.abs().clamp(max=100)) * 2.0 ** -22)
    if out.gate is not None:
        close(out.gate, G, eg)
        close(out.up, U, eu)


def check_backward(got, dh, x, wg, wu, gate_, up, act):
    X, Wg, Wu, dH, G, U = (t.double() for t in (x, wg, wu, dh, gate_, up))
    s, y, y1 = gate(G, act)
    err = (36 + y.abs().clamp(max=100)) * 2.0 ** -22
    dG = dH * U * s * (1 + G * y1 * (1 - s))
    eG = (dH * U).abs() * s * (1 + 2 * (G * y1).abs()) * err
    dU = dH * G * s
    eU = dU.abs() * err
    parts = []
    for d, e in ((dG, eG), (dU, eU)):
        if X.shape[0] <= 128:                            # sums of two bf16: 2^-9 of 2^-9
            parts.append((d, e + 2.0 ** -17 * d.abs()))
        else:
            parts.append((bf16(d), bf16(d + e) - bf16(d - e)))
    (dGr, sG), (dUr, sU) = parts
    dx, dwg, dwu = got
    if dx is not None:
        a = accumulation(2 * G.shape[1])
        close(dx, dGr @ Wg + dUr @ Wu, sG @ Wg.abs() + sU @ Wu.abs()
              + a * (dGr.abs() @ Wg.abs() + dUr.abs() @ Wu.abs()))
    if dwg is not None:
        a = accumulation(X.shape[0])
        for d, r, spread in ((dwg, dGr, sG), (dwu, dUr, sU)):
            close(d, r.t() @ X, spread.t() @ X.abs() + a * (r.abs().t() @ X.abs()))


SHAPES = [(1, 8, 8), (1, 64, 64), (3, 72, 200), (2, 520, 1000), (16, 256, 264), (17, 128, 2056),
          (128, 264, 96), (129, 136, 512), (255, 64, 16), (256, 512, 128), (300, 200, 1000),
          (1000, 1024, 2816), (2500, 72, 2000), (5000, 64, 520), (700, 8, 4104), (40, 4096, 304), (77, 600, 3000),
          (30, 128, 21000), (128, 64, 20000), (130, 72, 4104)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("pad", [0, 8])
@pytest.mark.parametrize("T,D,F", SHAPES, ids=[f"{t}x{d}x{f}" for t, d, f in SHAPES])
def test_both_passes_match_the_formulas(lib, gpu, T, D, F, pad, act):
    from paper_2608_15665_gb300 import firstorder as fo
    x, wg, wu = inputs(T, D, F, gpu, pad)
    out = fo.gated_linear(x, wg, wu, act, save=True)
    check_forward(out, x, wg, wu, act)
    alone = fo.gated_linear(x, wg, wu, act)
    assert alone.gate is None and torch.equal(alone.h, out.h)
    dh = make(T, F, gpu, 4, 0.1, pad)
    got = fo.gated_linear_backward(dh, x, wg, wu, out.gate, out.up, act)
    check_backward(got, dh, x, wg, wu, out.gate, out.up, act)
    # one side alone gives the same bits
    dx, none, _ = fo.gated_linear_backward(dh, x, wg, wu, out.gate, out.up, act, want_weights=False)
    assert none is None and torch.equal(dx, got[0])
    none, dwg, dwu = fo.gated_linear_backward(dh, x, wg, wu, out.gate, out.up, act, want_x=False)
    assert none is None and torch.equal(dwg, got[1]) and torch.equal(dwu, got[2])
    fo.gated_linear_sync()


@pytest.mark.parametrize("T,D,F,act", [(513, 2048, 4000, "silu"), (290, 3000, 11008, "gelu"),
                                       (777, 5120, 13824, "gelu"), (1100, 1024, 11008, "silu")])
def test_forward_in_several_rounds_of_tiles(lib, gpu, T, D, F, act):
    """Both kinds of tile, with one accumulator and with two, more tiles than SM pairs."""
    from paper_2608_15665_gb300 import firstorder as fo
    x, wg, wu = inputs(T, D, F, gpu)
    check_forward(fo.gated_linear(x, wg, wu, act, save=True), x, wg, wu, act)
    fo.gated_linear_sync()


def test_backward_in_several_rounds_of_tiles(lib, gpu):
    """More tiles of dX than SM pairs, and dW's dealt around the last ones; repeated, the same bits."""
    from paper_2608_15665_gb300 import firstorder as fo
    T, D, F = 2304, 4096, 1032
    x, wg, wu = inputs(T, D, F, gpu)
    out = fo.gated_linear(x, wg, wu, save=True)
    dh = make(T, F, gpu, 4, 0.1)
    runs = [fo.gated_linear_backward(dh, x, wg, wu, out.gate, out.up) for _ in range(6)]
    check_backward(runs[0], dh, x, wg, wu, out.gate, out.up, "silu")
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))
    fo.gated_linear_sync()


def test_results_in_rows_further_apart_leave_what_lies_between(lib, gpu):
    T, D, F, pad = 300, 136, 520, 16
    x, wg, wu = inputs(T, D, F, gpu, pad)
    outs = {n: torch.full((r, c + pad), 7.0, dtype=BF, device=gpu) for n, r, c in (
        ("H", T + 1, F), ("G", T + 1, F), ("U", T + 1, F), ("dX", T + 1, D), ("dWg", F + 1, D),
        ("dWu", F + 1, D))}
    cols = dict(H=F, G=F, U=F, dX=D, dWg=D, dWu=D)
    rows = dict(H=T, G=T, U=T, dX=T, dWg=F, dWu=F)
    v = {n: t[:rows[n], :cols[n]] for n, t in outs.items()}
    s = torch.cuda.current_stream()
    lib.zo_gated_forward(x, wg, wu, 0, v["H"], v["G"], v["U"], stream=s)
    dh = make(T, F, gpu, 4, 0.1, pad)
    ws = torch.empty(lib.zo_gated_workspace(T, D, F), dtype=torch.uint8, device=gpu)
    lib.zo_gated_backward(dh, x, wg, wu, 0, v["G"], v["U"], v["dX"], v["dWg"], v["dWu"], ws, stream=s)
    check_backward((v["dX"], v["dWg"], v["dWu"]), dh, x, wg, wu, v["G"], v["U"], "silu")
    for n, t in outs.items():
        assert (t[:, cols[n]:] == 7.0).all() and (t[rows[n]:] == 7.0).all(), n


def test_far_values_and_nan(lib, gpu):
    """Gates far out on either side, and what is not finite stays in its row or column."""
    from paper_2608_15665_gb300 import firstorder as fo
    x, wg, wu = inputs(64, 64, 64, gpu)
    for act in ("silu", "gelu"):
        big = (wg.float() * 60).to(BF)
        out = fo.gated_linear(x, big, wu, act, save=True)
        assert torch.isfinite(out.h).all()
        check_forward(out, x, big, wu, act)
        dh = make(64, 64, gpu, 4)
        got = fo.gated_linear_backward(dh, x, big, wu, out.gate, out.up, act)
        check_backward(got, dh, x, big, wu, out.gate, out.up, act)
        # gates as far as bf16 goes: the slope is 0 or 1
        g = torch.full((64, 64), 1e30, dtype=BF, device=gpu)
        g[::2] = -1e30
        g[1::4] = 100.0
        one = torch.ones_like(g)
        dx, dwg, dwu = fo.gated_linear_backward(one, x, wg, wu, g, one, act)
        want = (g > 0).double().t() @ x.double()
        assert float((dwg.double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) + 1e-6
        g[3, 4] = float("nan")
        dwg = fo.gated_linear_backward(one, x, wg, wu, g, one, act, want_x=False)[1]
        assert torch.isnan(dwg[4]).all() and torch.isfinite(dwg[:4]).all() and torch.isfinite(dwg[5:]).all()
    x2, wu2 = x.clone(), wu.clone()
    x2[5, 3], wu2[7, 2] = float("nan"), float("inf")
    h = fo.gated_linear(x2, wg, wu2).h
    bad = ~torch.isfinite(h)
    assert bad[5].all() and bad[:, 7].all()
    bad[5], bad[:, 7] = False, False
    assert not bad.any()


def test_no_tokens(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    _, wg, wu = inputs(1, 64, 72, gpu)
    x, h = torch.zeros(0, 64, dtype=BF, device=gpu), torch.zeros(0, 72, dtype=BF, device=gpu)
    assert fo.gated_linear(x, wg, wu, save=True).gate.shape == (0, 72)
    dx, dwg, dwu = fo.gated_linear_backward(h, x, wg, wu, h, h)
    assert dx.shape == (0, 64) and (dwg == 0).all() and (dwu == 0).all() and dwg.shape == (72, 64)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_autograd_gives_the_gradients_and_they_are_difference_quotients(lib, gpu, act):
    from paper_2608_15665_gb300 import firstorder as fo
    x, wg, wu = inputs(33, 72, 104, gpu)
    leaves = [t.clone().requires_grad_() for t in (x, wg, wu)]
    dh = make(33, 104, gpu, 4)
    fo.GatedLinear.apply(*leaves, act).backward(dh)
    out = fo.gated_linear(x, wg, wu, act, save=True)
    want = fo.gated_linear_backward(dh, x, wg, wu, out.gate, out.up, act)
    assert all(torch.equal(a.grad, b) for a, b in zip(leaves, want))
    # inputs and gradients in other orders and places are taken as copies
    base = torch.zeros(33 * 72 + 3, dtype=BF, device=gpu)
    for odd in (x.t().contiguous().t(), base[3:].view(33, 72).copy_(x)):
        leaf = odd.detach().requires_grad_()
        h = fo.GatedLinear.apply(leaf, wg, wu, act)
        h.backward(dh.t().contiguous().t())
        assert torch.equal(h, out.h) and torch.equal(leaf.grad, want[0])
    # along a direction, in 64 bits: the sum of gradient times direction, to bf16's grade
    dirs = [make(*t.shape, gpu, 9 + i).double() for i, t in enumerate((x, wg, wu))]

    def f(h):
        X, Wg, Wu = (t.double() + h * d for t, d in zip((x, wg, wu), dirs))
        G = X @ Wg.t()
        return float((G * gate(G, act)[0] * (X @ Wu.t()) * dh.double()).sum())
    quotient = (f(1e-4) - f(-1e-4)) / 2e-4
    total = sum(float((a.double() * d).sum()) for a, d in zip(want, dirs))
    size = sum(float((a.double() * d).square().sum()) for a, d in zip(want, dirs)) ** 0.5
    assert abs(total - quotient) <= 2.0 ** -6 * size
    # what is not asked for is not made; a second derivative is refused
    leaf = x.clone().requires_grad_()
    fo.GatedLinear.apply(leaf, wg, wu, act).backward(dh)
    assert torch.equal(leaf.grad, want[0])
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(fo.GatedLinear.apply(leaf, wg, wu, act), leaf, dh, create_graph=True)
        g.sum().backward()


def test_capture_replay_and_other_streams(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    data = [inputs(200, 128, 264, gpu)[0], make(200, 128, gpu, 8)]
    _, wg, wu = inputs(200, 128, 264, gpu)
    dh = make(200, 264, gpu, 4)

    def both(x):
        out = fo.gated_linear(x, wg, wu, save=True)
        return (out.h, *fo.gated_linear_backward(dh, x, wg, wu, out.gate, out.up))
    want = [both(x) for x in data]
    buf = data[0].clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = both(buf)
    for i in (1, 0):
        buf.copy_(data[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        buf.copy_(data[1])
        got = both(buf)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))
    fo.gated_linear_sync()
