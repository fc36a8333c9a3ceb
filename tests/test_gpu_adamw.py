"""The AdamW step on the GPU against its formulas in 64 bits, on the same inputs.

Tolerances, per element, derived before the first run.  u = 2^-24.  m and v are two products
and a sum: 3 u of the sum of magnitudes (4 u for v, whose g^2 is a product more).  W's update
divides m c by r c' + eps: with the hardware's approximate division and root (2 ulp each), the
corrections rounded to fp32 (2 u each) and the products, 24 u of the update's magnitude and 2 u of
W's; the update's own inputs are off by m's 3 u of its magnitudes and r's 2 u.  Then half an ulp
of a bf16 W: 2^-8 of it at most.

A code of 8 bits is floor(x + r) with x in steps and r the random part.  x is off by m's error
above, the scaling's 2^-20 of a step and the root's 2^-22 of itself: with |x| < 16 steps by less
than 2^-17 for terms without cancellation, so the code is the one of 64 bits where x + r is
further than that from a whole number (scaled with the cancellation of m), else one of two."""

import numpy as np
import pytest
import torch

from oracle import rng

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
B1, B2, EPS, LR, WD = 0.9, 0.999, 1e-8, 1e-2, 0.1


def f64(t):
    return t.detach().float().cpu().double().numpy()


def strided(x, dtype, dev, pad):
    """x (2-D) in `dtype` in rows `pad` elements apart, or contiguous."""
    buf = torch.full((x.shape[0], x.shape[1] + pad), float("nan"))
    buf[:, :x.shape[1]] = x
    return buf.to(dtype).to(dev)[:, :x.shape[1]]


def make(shape, dtype, gdtype, dev, seed, pad=0, offset=0):
    """W, G: `offset` elements into their buffers."""
    g = torch.Generator().manual_seed(seed)
    n = int(np.prod(shape))

    def one(scale, dt):
        x = torch.randn(shape, generator=g) * scale
        if pad:
            return strided(x, TYPES[dt], dev, pad)
        buf = torch.full((n + offset,), float("nan"))
        buf[offset:] = x.flatten()
        return buf.to(TYPES[dt]).to(dev)[offset:].view(shape)
    return one(0.02, dtype), one(1e-3, gdtype)


def formulas(W, G, m, v, t):
    """(W, m, v, magnitudes of m's and of W's error terms)"""
    m1 = B1 * m + (1 - B1) * G
    v1 = B2 * v + (1 - B2) * G * G
    den = np.sqrt(v1 / (1 - B2 ** t)) + EPS
    upd = LR * m1 / (1 - B1 ** t) / den
    mm = B1 * np.abs(m) + (1 - B1) * np.abs(G)
    W1 = (1 - LR * WD) * W - upd
    lim = 2 * U * np.abs(W) + U * (24 + 4) * np.abs(upd) + 3 * U * LR * mm / (1 - B1 ** t) / den
    return W1, m1, v1, mm, lim


def check_w(got, want, lim, dtype):
    half = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want)
    assert np.all(np.abs(f64(got) - want) <= lim + half * 1.01)


SHAPES = [(1,), (7,), (8,), (255,), (256,), (257,), (4096,), (4097,), (33, 100), (3, 5, 7), (8, 5120)]


@pytest.mark.parametrize("dtype,gdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                          ("f32", "bf16")])
@pytest.mark.parametrize("t", [1, 2, 1000])
def test_step_of_many_tensors_in_32_bits(lib, gpu, dtype, gdtype, t):
    from paper_2608_15665_gb300 import firstorder as fo
    W, G = zip(*[make(s, dtype, gdtype, gpu, i, offset=i % 3) for i, s in enumerate(SHAPES)])
    W, G = list(W), list(G)
    pads = [make((9, 70), dtype, gdtype, gpu, 50, pad=3), make((300, 8), dtype, gdtype, gpu, 51, pad=8)]
    empty = make((0,), dtype, gdtype, gpu, 52)
    for w, g in pads + [empty]:
        W.append(w)
        G.append(g)
    states = [fo.adamw_state(w) for w in W]
    g = torch.Generator().manual_seed(5)
    for s in states:
        s.m.copy_(torch.randn(s.m.shape, generator=g) * 1e-3)
        s.v.copy_(torch.rand(s.v.shape, generator=g) * 1e-6)
    before = [(f64(w), f64(x), f64(s.m).reshape(w.shape), f64(s.v).reshape(w.shape))
              for w, x, s in zip(W, G, states)]
    gaps = [w._base.clone() for w, _ in pads]
    opt = fo.AdamW(W, G, states)
    opt.step(LR, (B1, B2), EPS, WD, t=t)
    torch.cuda.synchronize()
    for w, s, b in zip(W, states, before):
        want, m1, v1, mm, lim = formulas(*b, t)
        check_w(w, want, lim, dtype)
        assert np.all(np.abs(f64(s.m).reshape(w.shape) - m1) <= 3 * U * mm)
        assert np.all(np.abs(f64(s.v).reshape(w.shape) - v1) <= 4 * U * v1)
    for (w, _), old in zip(pads, gaps):                # what lies between the rows stays
        n = w.shape[1]
        assert torch.equal(w._base[:, n:].view(torch.uint8), old[:, n:].view(torch.uint8))
    assert opt.steps == t


def values(codes, exps, shape):
    """64-bit values of an 8-bit state."""
    e = np.repeat(np.maximum(exps.cpu().numpy().astype(np.int64), 40) - 134, 256)[:codes.numel()]
    return (f64(codes) * 2.0 ** e).reshape(shape)


def random_of(seed, index, t, n):
    words = rng.philox_block(seed, index, t, 6 << 24, -(-n // 8) * 4).astype(np.uint64)
    halves = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 1).reshape(-1)
    return halves[:n].astype(np.float64) / 65536.0


def check_codes(codes, exps, x, top, r, err, positive):
    """codes of x (flat, 64 bits; off by at most err) against floor(x + r) in steps."""
    n = x.size
    pad = np.zeros(-(-n // 256) * 256)
    pad[:n] = top
    biggest = pad.reshape(-1, 256).max(1)
    E = np.where(biggest > 0, np.floor(np.log2(np.maximum(biggest, 1e-300))) + 127, 0)
    got = exps.cpu().numpy().astype(np.int64)
    near = np.abs(np.log2(np.maximum(biggest, 1e-300)) - np.round(np.log2(np.maximum(biggest, 1e-300)))) < 1e-6
    assert np.all((got == E) | near & (np.abs(got - E) == 1))
    s = 2.0 ** (134.0 - np.repeat(np.maximum(got, 40), 256)[:n])
    y, off = np.abs(x) * s, err * s
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(y, 1e-30))), -6) - 3)
    # (a value next to a power of two may be taken from either side of it)
    p = y / step + r
    slack = off / step + 2.0 ** -19
    lo, hi = np.floor(p - slack) * step, np.floor(p + slack) * step
    if positive:
        lo, hi = np.where(x > 0, np.maximum(lo, 2.0 ** -9), lo), np.where(x > 0, np.maximum(hi, 2.0 ** -9), hi)
    c = f64(codes).reshape(-1)
    assert np.all((np.abs(c) >= lo) & (np.abs(c) <= hi))
    assert np.all((c == 0) | (np.sign(c) == np.sign(x)))
    return float(np.mean(lo != hi))


@pytest.mark.parametrize("dtype,gdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_steps_in_8_bits(lib, gpu, dtype, gdtype):
    from paper_2608_15665_gb300 import firstorder as fo
    W, G = zip(*[make(s, dtype, gdtype, gpu, i, offset=i % 2) for i, s in enumerate(SHAPES)])
    W, G = list(W), list(G)
    w, g = make((9, 70), dtype, gdtype, gpu, 50, pad=3)
    W.append(w)
    G.append(g)
    opt = fo.AdamW(W, G, bits=8, seed=(5 << 32) + 77)
    for t in range(1, 5):
        before = [(f64(w), f64(x), values(s.m, s.m_exp, w.shape), values(s.v, s.v_exp, w.shape) ** 2)
                  for w, x, s in zip(W, G, opt.states)]
        opt.step(LR, (B1, B2), EPS, WD)
        torch.cuda.synchronize()
        unsure = []
        for i, (w, s, b) in enumerate(zip(W, opt.states, before)):
            want, m1, v1, mm, lim = formulas(*b, t)
            check_w(w, want, lim, dtype)
            r = random_of((5 << 32) + 77, i, t, w.numel())
            root = np.sqrt(v1).reshape(-1)
            unsure.append(check_codes(s.m, s.m_exp, m1.reshape(-1), np.abs(m1).reshape(-1), r,
                                      3 * U * mm.reshape(-1), False))
            unsure.append(check_codes(s.v, s.v_exp, root, root, r, 6 * U * root, True))
        assert max(unsure[-1:]) < 1e-2 and np.mean(unsure) < 1e-2
        for k, x in enumerate(G):                      # other gradients in the next step
            x.mul_(-0.7 if k % 2 else 1.6)
    opt.close()


def test_8_bit_means_follow_the_32_bit_ones(lib, gpu):
    """Running means that move by a thousandth a step: v of 2^16 elements from zero under gradients
    of unit variance stays within its noise, and decays under zero ones."""
    from paper_2608_15665_gb300 import firstorder as fo
    n = 1 << 16
    W = torch.zeros(n, device=gpu)
    G = torch.zeros(n, device=gpu)
    opt = fo.AdamW([W], [G], bits=8, seed=3)
    ref = fo.AdamW([torch.zeros(n, device=gpu)], [G])
    g = torch.Generator(device=gpu).manual_seed(1)

    def root():
        return torch.from_numpy(values(opt.states[0].v, opt.states[0].v_exp, (n,)))
    for _ in range(1500):
        G.copy_(torch.randn(n, generator=g, device=gpu))
        opt.step(0.0)
        ref.step(0.0)
    r, want = root(), ref.states[0].v.double().cpu().sqrt()
    # r's steps are 1/16 to 1/8 of it and are taken up or down: the variance a step is at most
    # |dr| r / 8 with |dr| ~ r (1 - b2) / 2 |g^2 / v - 1|, mean magnitude 0.97, and v forgets it at
    # the rate 2 (1 - b2): at most sqrt(0.97 / 32) = 0.17 of r; the mean of r^2 exceeds v by as
    # much as that variance
    rel = (r - want) / want
    assert float(rel.std()) < 0.19
    assert abs(float(rel.mean())) < 0.04
    # (v takes sixteen codes of a power of two, not one of them alone)
    assert len(torch.unique(opt.states[0].v.float())) > 8
    G.zero_()
    for _ in range(700):
        opt.step(0.0)
        ref.step(0.0)
    r2, want2 = root(), ref.states[0].v.double().cpu().sqrt()
    assert abs(float((r2 / want2).mean()) - 1) < 0.06


def test_nothing_but_its_own_element_sees_an_infinity_or_nan(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    for bits in (32, 8):
        W, G = make((1000,), "f32", "f32", gpu, 1)
        G2 = G.clone()
        G2[5], G2[300], G2[999] = float("inf"), float("nan"), float("-inf")
        W2 = W.clone()
        a, b = fo.AdamW([W], [G], bits=bits), fo.AdamW([W2], [G2], bits=bits)
        a.step(LR)
        b.step(LR)
        at = torch.tensor([5, 300, 999], device=gpu)
        keep = torch.ones(1000, dtype=torch.bool, device=gpu)
        keep[at] = False
        assert torch.isnan(W2[at]).all() and torch.equal(W[keep], W2[keep])
        m = b.states[0].m.float()
        assert torch.isnan(m[at]).sum() == (1 if bits == 32 else 3) and torch.isfinite(m[keep]).all()


def test_zero_gradients_and_zero_states_leave_weights_but_for_decay(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    for bits in (32, 8):
        W, G = make((700,), "f32", "f32", gpu, 1)
        G.zero_()
        want = f64(W) * (1 - LR * WD)
        opt = fo.AdamW([W], [G], bits=bits)
        opt.step(LR, weight_decay=WD)
        assert np.all(np.abs(f64(W) - want) <= 2 * U * np.abs(want))
        # gradients far below the block's largest, and later zero: no update without a second moment
        G[0] = 1e6
        G[1:] = 1e-9
        opt.step(LR, weight_decay=0.0)
        before = W.clone()
        G.zero_()
        opt.step(LR, weight_decay=0.0)
        assert float((W - before).abs().max()) < 20 * LR


def test_a_count_on_the_device_and_a_replayed_graph(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    for bits in (32, 8):
        W, G = make((5000,), "f32", "f32", gpu, 1)
        W2, G2 = W.clone(), G.clone()
        want = fo.AdamW([W], [G], bits=bits, seed=9)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            count = torch.zeros(1, dtype=torch.int64, device=gpu)
            opt = fo.AdamW([W2], [G2], bits=bits, seed=9, count=count)
            opt.step(LR)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            opt.step(LR)
            with pytest.raises(lib.ZoError):            # without a count: the same number every time
                want.step(LR)
        want.step(LR)
        for k in range(3):
            for x in (G, G2):
                x.mul_(-0.5)
            want.step(LR)
            graph.replay()
        torch.cuda.synchronize()
        assert int(count) == 4 and want.steps == 4
        # 1 - b^t is rounded from 64 bits in both
        assert float((W - W2).abs().max()) <= 8 * U * LR * 4
        assert torch.equal(want.states[0].m.view(torch.uint8), opt.states[0].m.view(torch.uint8))


def test_steps_under_another_stream_are_ordered(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    out = []
    for side in (False, True):
        W, G = make((100000,), "bf16", "bf16", gpu, 1)
        fresh = G.clone()
        opt = fo.AdamW([W], [torch.zeros_like(G)], bits=8)
        torch.cuda.synchronize()
        s = torch.cuda.Stream() if side else torch.cuda.current_stream()
        with torch.cuda.stream(s):
            torch.cuda._sleep(50_000_000)
            opt.grads[0].copy_(fresh)
            opt.step(LR)
            out.append(W.clone())
        torch.cuda.synchronize()
    assert torch.equal(*out)


def test_the_same_steps_give_the_same_bits(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    out = []
    for _ in range(2):
        W, G = make((300000,), "bf16", "bf16", gpu, 1)
        opt = fo.AdamW([W], [G], bits=8, seed=4)
        for _ in range(3):
            opt.step(LR)
        out.append((W, opt.states[0].m.view(torch.uint8), opt.states[0].v.view(torch.uint8)))
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_refusals_of_a_step(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    W, G = make((100,), "f32", "f32", gpu, 1)
    before = W.clone()
    opt = fo.AdamW([W], [G])
    for kw in (dict(t=0), dict(t=-1), dict(lr=float("nan")), dict(betas=(1.0, 0.9)),
               dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(weight_decay=float("inf"))):
        args = dict(lr=LR)
        args.update(kw)
        with pytest.raises(lib.ZoError):
            opt.step(**args)
    counted = fo.AdamW([W], [G], count=torch.zeros(1, dtype=torch.int64, device=gpu))
    with pytest.raises(lib.ZoError):
        counted.step(LR, t=3)
    with pytest.raises(lib.ZoError):
        fo.AdamW([W, W], [G, G])
    torch.cuda.synchronize()
    assert torch.equal(W, before) and opt.steps == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_exponents_are_those_of_sums_of_rounded_products(lib, gpu, dtype):
    """Codes and bf16 gradients have few digits: the sums often meet a power of two, and then a fused
    product's other rounding shows in the block's exponent.  Bit for bit against fp32 arithmetic."""
    from paper_2608_15665_gb300 import firstorder as fo
    f = np.float32
    n = 1 << 21
    g = torch.Generator().manual_seed(3)
    W = torch.zeros(n, dtype=TYPES[dtype], device=gpu)
    G = (torch.randn(n, generator=g) * 2.0 ** torch.randint(-12, 12, (n,), generator=g).float())
    G = G.to(torch.bfloat16).to(TYPES[dtype]).to(gpu)
    state = fo.adamw_state(W, 8)
    codes = torch.randint(0, 0x7F, (n,), generator=g, dtype=torch.uint8)
    state.m.view(torch.uint8).copy_(codes)
    state.v.view(torch.uint8).copy_(codes.flip(0))
    for e in (state.m_exp, state.v_exp):
        e.copy_(torch.randint(115, 140, e.shape, generator=g).to(torch.uint8))
    m = values(state.m, state.m_exp, (n,)).astype(f)
    r = values(state.v, state.v_exp, (n,)).astype(f)
    x = f64(G).astype(f)
    opt = fo.AdamW([W], [G], [state], bits=8)
    opt.step(LR, (B1, B2), EPS, WD, t=7)
    torch.cuda.synchronize()
    m1 = f(B1) * m + f(1.0 - B1) * x
    v1 = f(B2) * (r * r) + f(1.0 - B2) * (x * x)
    top = np.abs(m1).reshape(-1, 256).max(1)
    em = np.where(top > 0, np.frexp(top)[1] + 126, 0)
    ev = np.frexp(v1.reshape(-1, 256).max(1))[1] - 1
    assert np.array_equal(state.m_exp.cpu().numpy(), em)
    assert np.array_equal(state.v_exp.cpu().numpy(), (ev >> 1) + 127)
    # and so are the codes (those of normal numbers: below, products are rounded once more)
    u = random_of(0, 0, 7, n)
    for code, x, E in ((state.m, np.abs(m1), em), (state.v, np.sqrt(v1), (ev >> 1) + 127)):
        y = x.astype(np.float64) * 2.0 ** np.repeat(134.0 - np.maximum(E, 40), 256)
        step = 2.0 ** (np.floor(np.log2(np.maximum(y, 1e-30))) - 3)
        normal = y >= 2.0 ** -6
        assert np.array_equal(np.abs(f64(code))[normal], (np.floor(y / step + u) * step)[normal])
