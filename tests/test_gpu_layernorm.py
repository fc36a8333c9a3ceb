"""Layer normalisation on the GPU against its formulas in 64 bits, on the same inputs.

Tolerances, per element, derived before the first run.  u = 2^-24.  A sum of n fp32 terms,
taken over at least 32 lanes and a tree, errs by at most (n / 32 + 20) u of the sum of
magnitudes; its statistical error is far less.  With S = max |h - mean| rstd of a row (at
most sqrt(n)) the chain (h - mean) rstd w + b adds a few roundings, each at the scale of its
operands: |h| rstd |w|, |mean| rstd |w|, |y|, |b|.  So

  |y - y_64|  <= (n / 32 + 40) u (|w| rstd (|h| + mean_j |h_j|) + |xh w| + |b|) + half an ulp

and the backward pass likewise with the magnitudes of its own terms.  Half an ulp of a bf16
output is 2^-8 of it at most (2^-9 above its power of two), taken with a guard for a result
that lands across a rounding boundary."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows_of(rows, cols, dtype, dev, seed, pad=0, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((rows, cols + pad), float("nan"))
    buf[:, :cols] = torch.randn(rows, cols, generator=g) * scale + shift
    return buf.to(TYPES[dtype]).to(dev)[:, :cols]


def vec(n, dtype, dev, seed, center):
    g = torch.Generator().manual_seed(seed)
    return (center + 0.3 * torch.randn(n, generator=g)).to(TYPES[dtype]).to(dev)


def f64(t):
    return t.detach().float().cpu().double().numpy()


def grade(n):
    return (n / 32 + 40) * U


def rounding(dtype, v):
    return (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * np.abs(v)


def stats(h, eps):
    mean = h.mean(1, keepdims=True)
    var = ((h - mean) ** 2).mean(1, keepdims=True)
    return mean, 1.0 / np.sqrt(var + eps)


# rows, columns, padding of the rows, offset of the mean
SHAPES = [(1, 1, 0, 0.0), (3, 7, 0, 0.0), (5, 64, 0, 0.0), (2, 129, 3, 0.0), (33, 512, 0, 0.0),
          (9, 513, 0, 0.0), (4, 768, 8, 100.0), (6, 1001, 0, 0.0), (3, 2048, 0, 0.0),
          (2, 4100, 4, 0.0), (5, 5120, 0, 0.0), (2, 8192, 0, -30.0), (2, 11008, 0, 0.0),
          (3, 16384, 0, 0.0), (2, 16392, 0, 0.0), (1, 33001, 0, 0.0), (700, 96, 0, 0.0),
          (650, 1536, 0, 0.0)]


@pytest.mark.parametrize("dtype,wdtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"),
                                          ("f32", "bf16")])
@pytest.mark.parametrize("rows,cols,pad,shift", SHAPES, ids=[f"{s[0]}x{s[1]}" for s in SHAPES])
def test_both_passes_match_the_formulas(lib, gpu, rows, cols, pad, shift, dtype, wdtype):
    from paper_2608_15665_gb300 import firstorder as fo
    eps = 1e-5
    x = rows_of(rows, cols, dtype, gpu, 1, pad, shift=shift)
    w, b = vec(cols, wdtype, gpu, 2, 1.0), vec(cols, wdtype, gpu, 3, 0.0)
    dy = rows_of(rows, cols, dtype, gpu, 4, pad)
    out = fo.layer_norm(x, w, b, eps)
    dx, dw, db = fo.layer_norm_backward(dy, x, w, out.mean, out.rstd)
    assert out.h is None
    check_forward(out, f64(x), w, b, eps, dtype)
    check_backward(dx, dw, db, f64(dy), f64(x), w, f64(out.mean), f64(out.rstd), 0.0, dtype,
                   wdtype)


def check_forward(out, h, w, b, eps, dtype):
    n = h.shape[1]
    mean, rstd = stats(h, eps)
    W = np.ones(n) if w is None else f64(w)
    B = np.zeros(n) if b is None else f64(b)
    xh = (h - mean) * rstd
    y = xh * W + B
    size = np.abs(h).mean(1, keepdims=True)
    lim = grade(n) * (np.abs(W) * rstd * (np.abs(h) + size) + np.abs(xh * W) + np.abs(B))
    assert np.all(np.abs(f64(out.y) - y) <= lim + rounding(dtype, y))
    if out.mean is not None:
        assert np.all(np.abs(f64(out.mean)[:, None] - mean) <= grade(n) * size)
        # rstd's error: the variance's, of terms (h - mean)^2 whose own error is that of mean
        rel = grade(n) * (1 + size * rstd) + 4 * U
        assert np.all(np.abs(f64(out.rstd)[:, None] / rstd - 1) <= rel)


def check_backward(dx, dw, db, dy, h, w, mean, rstd, dr, dtype, wdtype):
    rows, n = h.shape
    W = np.ones(n) if w is None else f64(w)
    mean, rstd = mean[:, None], rstd[:, None]
    xh, g = (h - mean) * rstd, dy * W
    want = rstd * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True)) + dr
    xs = (np.abs(h) + np.abs(mean)) * rstd                     # xh's operands
    mag = rstd * (np.abs(g) + np.abs(g).mean(1, keepdims=True) +
                  xs * (np.abs(g) * xs).mean(1, keepdims=True)) + np.abs(dr)
    assert np.all(np.abs(f64(dx) - want) <= grade(n) * mag + rounding(dtype, want))
    if dw is not None:
        # a chain over the rows of one CTA, then one over the CTAs
        want, mag = (dy * xh).sum(0), (np.abs(dy) * xs).sum(0)
        assert np.all(np.abs(f64(dw) - want) <= (rows + 40) * U * mag + rounding(wdtype, want))
    if db is not None:
        want, mag = dy.sum(0), np.abs(dy).sum(0)
        assert np.all(np.abs(f64(db) - want) <= (rows + 40) * U * mag + rounding(wdtype, want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", [(4, 256, 0), (5, 1000, 8), (3, 1001, 1), (2, 20000, 0)])
def test_residual(lib, gpu, rows, cols, pad, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    x, r = rows_of(rows, cols, dtype, gpu, 1, pad), rows_of(rows, cols, dtype, gpu, 5, pad, 2.0)
    w, b = vec(cols, dtype, gpu, 2, 1.0), vec(cols, dtype, gpu, 3, 0.0)
    out = fo.layer_norm(x, w, b, 1e-5, residual=r)
    assert torch.equal(out.h, (x.float() + r.float()).to(TYPES[dtype]))
    check_forward(out, f64(out.h), w, b, 1e-5, dtype)
    dy, dr = rows_of(rows, cols, dtype, gpu, 6, pad), rows_of(rows, cols, dtype, gpu, 7, pad)
    dx, dw, db = fo.layer_norm_backward(dy, out.h, w, out.mean, out.rstd, dresidual=dr)
    check_backward(dx, dw, db, f64(dy), f64(out.h), w, f64(out.mean), f64(out.rstd), f64(dr),
                   dtype, dtype)


@pytest.mark.parametrize("cols", [100, 2048, 40000])
def test_optional_parts(lib, gpu, cols):
    from paper_2608_15665_gb300 import firstorder as fo
    x, dy = rows_of(6, cols, "f32", gpu, 1), rows_of(6, cols, "f32", gpu, 2)
    out = fo.layer_norm(x, None, None, 1e-5)
    check_forward(out, f64(x), None, None, 1e-5, "f32")
    bare = fo.layer_norm(x, None, None, 1e-5, stats=False)
    assert bare.mean is None and torch.equal(bare.y, out.y)
    b = vec(cols, "f32", gpu, 3, 0.0)
    check_forward(fo.layer_norm(x, None, b, 1e-5), f64(x), None, b, 1e-5, "f32")
    for want_w, want_b in ((True, True), (True, False), (False, True), (False, False)):
        dx, dw, db = fo.layer_norm_backward(dy, x, None, out.mean, out.rstd, want_weight=want_w,
                                            want_bias=want_b)
        assert (dw is not None, db is not None) == (want_w, want_b)
        check_backward(dx, dw, db, f64(dy), f64(x), None, f64(out.mean), f64(out.rstd), 0.0,
                       "f32", "f32")


def test_no_rows_give_zero_gradients(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    x = torch.empty(0, 48, device=gpu)
    out = fo.layer_norm(x, torch.ones(48, device=gpu), None)
    dx, dw, db = fo.layer_norm_backward(x, x, torch.ones(48, device=gpu), out.mean, out.rstd)
    torch.cuda.synchronize()
    assert out.y.shape == dx.shape == (0, 48)
    assert float(dw.abs().max()) == float(db.abs().max()) == 0.0


@pytest.mark.parametrize("cols", [96, 3001, 20001])
def test_constant_rows_and_rows_that_are_not_finite(lib, gpu, cols):
    from paper_2608_15665_gb300 import firstorder as fo
    x = rows_of(5, cols, "f32", gpu, 1)
    x[1] = 3.25                                            # no spread: y = bias exactly
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    w, b = vec(cols, "f32", gpu, 2, 1.0), vec(cols, "f32", gpu, 3, 0.0)
    out = fo.layer_norm(x, w, b, 1e-5)
    assert torch.equal(out.y[1], b) and float(out.rstd[1]) == pytest.approx(1e-5 ** -0.5, rel=1e-6)
    assert bool(torch.isnan(out.y[2]).all()) and bool(torch.isnan(out.y[3]).all())
    keep = [0, 4]
    rest = fo.layer_norm(x[keep].contiguous(), w, b, 1e-5)
    assert torch.equal(out.y[keep], rest.y)                # the other rows are untouched
    dx, dw, db = fo.layer_norm_backward(torch.ones_like(x), x, w, out.mean, out.rstd)
    assert bool(torch.isfinite(dx[[0, 1, 4]]).all()) and bool(torch.isnan(dx[2:4]).any(1).all())


@pytest.mark.parametrize("rows,cols,dtype", [(257, 520, "bf16"), (40, 5120, "bf16"),
                                             (130, 77, "f32"), (4000, 256, "bf16")])
def test_repeats_and_back_to_back_calls_give_the_same_bits(lib, gpu, rows, cols, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    x, dy = rows_of(rows, cols, dtype, gpu, 1), rows_of(rows, cols, dtype, gpu, 2)
    w, b = vec(cols, dtype, gpu, 3, 1.0), vec(cols, dtype, gpu, 4, 0.0)
    first = None
    for _ in range(4):
        out = fo.layer_norm(x, w, b)
        again = fo.layer_norm(out.y, w, b)                 # reads what the call before writes
        got = (out.y, again.y) + fo.layer_norm_backward(dy, x, w, out.mean, out.rstd)
        first = first or got
        assert all(torch.equal(p, q) for p, q in zip(first, got))


def test_a_stream_of_ones_own(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    x = rows_of(300, 4096, "bf16", gpu, 1)
    w, b = vec(4096, "f32", gpu, 3, 1.0), vec(4096, "f32", gpu, 4, 0.0)
    want = fo.layer_norm(x, w, b).y
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        z = x.float().mul(1.0).to(torch.bfloat16)          # made on that stream
        got = fo.layer_norm(z, w, b).y
    s.synchronize()
    assert torch.equal(want, got)


def test_padding_is_not_written(lib, gpu):
    x = rows_of(7, 130, "bf16", gpu, 1, pad=6)
    buf = torch.full((7, 136), 7.0, dtype=torch.bfloat16, device=gpu)
    lib.zo_layernorm_forward(x, None, None, None, 1e-5, buf[:, :130], stream=None)
    torch.cuda.synchronize()
    assert bool((buf[:, 130:] == 7.0).all()) and not bool((buf[:, :130] == 7.0).any())


def test_gradients_match_differences(lib, gpu):
    """Central differences of L = sum(c y) in 64 bits at step h: the formula's gradient plus
    O(h^2) = 1e-8 of the third derivative, which at these sizes is a few units."""
    from paper_2608_15665_gb300 import firstorder as fo
    rows, n, h = 3, 24, 1e-4
    x, c = rows_of(rows, n, "f32", gpu, 1), rows_of(rows, n, "f32", gpu, 2)
    w, b = vec(n, "f32", gpu, 3, 1.0), vec(n, "f32", gpu, 4, 0.0)

    def loss(X, Wt, Bs):
        m, r = stats(X, 1e-5)
        return float((f64(c) * ((X - m) * r * Wt + Bs)).sum())

    xs = [t.clone().requires_grad_() for t in (x, w, b)]
    (fo.LayerNorm.apply(xs[0], xs[1], xs[2], 1e-5) * c).sum().backward()
    base = [f64(x), f64(w), f64(b)]
    for k, t in enumerate(xs):
        num = np.zeros_like(base[k])
        for i in np.ndindex(num.shape):
            at = [a.copy() for a in base]
            at[k][i] += h
            up = loss(*at)
            at[k][i] -= 2 * h
            num[i] = (up - loss(*at)) / (2 * h)
        assert np.abs(f64(t.grad) - num).max() <= 2e-5 * max(1.0, np.abs(num).max())


def test_the_workspace_is_checked(lib, gpu):
    x = torch.zeros(4, 64, device=gpu)
    v = torch.zeros(64, device=gpu)
    st = torch.zeros(4, device=gpu)
    need = lib.zo_layernorm_workspace(4, 64)
    assert need > 0
    for ws in (None, torch.empty(need - 1, dtype=torch.uint8, device=gpu)):
        with pytest.raises(lib.ZoError) as e:
            lib.zo_layernorm_backward(x, x, None, v, st, st, torch.empty_like(x), v, v, ws)
        assert e.value.status == lib.ZO_ERR_INVALID_ARG


# more rows than are in flight at once, on and off 16-byte boundaries
MANY = [(2000, 77, 0), (1900, 1003, 1), (2500, 640, 0), (700, 2051, 0), (900, 2048, 8),
        (330, 5121, 0), (400, 5120, 0), (340, 9001, 2), (320, 12288, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,cols,pad", MANY, ids=[f"{s[0]}x{s[1]}" for s in MANY])
def test_many_rows(lib, gpu, rows, cols, pad, residual, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    x, dy = rows_of(rows, cols, dtype, gpu, 1, pad), rows_of(rows, cols, dtype, gpu, 4, pad)
    r = rows_of(rows, cols, dtype, gpu, 5, 0) if residual else None
    dr = rows_of(rows, cols, dtype, gpu, 6, pad) if residual else None
    w, b = vec(cols, "f32", gpu, 2, 1.0), vec(cols, "f32", gpu, 3, 0.0)
    out = fo.layer_norm(x, w, b, 1e-5, residual=r)
    h = out.h if residual else x
    if residual:
        assert torch.equal(out.h, (x.float() + r.float()).to(TYPES[dtype]))
    check_forward(out, f64(h), w, b, 1e-5, dtype)
    dx, dw, db = fo.layer_norm_backward(dy, h, w, out.mean, out.rstd, dresidual=dr)
    check_backward(dx, dw, db, f64(dy), f64(h), w, f64(out.mean), f64(out.rstd),
                   f64(dr) if residual else 0.0, dtype, "f32")


@pytest.mark.parametrize("lead", [1, 3, 5])
def test_rows_that_start_anywhere(lib, gpu, lead):
    """Views whose first element lies at an odd place of its buffer: a row's first and last 16
    bytes are shared with values that are not the row's (NaN here)."""
    from paper_2608_15665_gb300 import firstorder as fo
    rows, cols = 2100, 250
    base = torch.full((rows * 260 + 16,), float("nan"), dtype=torch.bfloat16, device=gpu)
    x = torch.as_strided(base, (rows, cols), (260, 1), lead)
    x.copy_(rows_of(rows, cols, "bf16", gpu, 9))
    w, b = vec(cols, "bf16", gpu, 2, 1.0), vec(cols, "bf16", gpu, 3, 0.0)
    out = fo.layer_norm(x, w, b)
    plain = fo.layer_norm(x.contiguous(), w, b)
    assert torch.equal(out.y, plain.y) and torch.equal(out.mean, plain.mean)
    dy = rows_of(rows, cols, "bf16", gpu, 4)
    got = fo.layer_norm_backward(dy, x, w, out.mean, out.rstd)
    check_backward(*got, f64(dy), f64(x), w, f64(out.mean), f64(out.rstd), 0.0, "bf16", "bf16")
