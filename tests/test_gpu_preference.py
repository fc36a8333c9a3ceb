"""The preference loss on the GPU against its formulas in 64 bits, on the same inputs.

Tolerances, derived before the first run.  u = 2^-24.  A row's sum of V terms e^d, d = l - top, goes
over 256 threads and a tree: (V / 256 + 60) u of it, and each term is off by the hardware's 2^-22
and by |d| 2 u from its exponent's roundings.  So lse is off by that share of the sum, and by its
own rounding; logp by the same share and its rounding.  Sequence sums add no error of note in 64
bits, but for their rounding.  A gradient scale (hit - p) is off by scale p (|l - lse| 2 u + 8 u +
lse's error), three roundings of the result, and half an ulp (bf16: 2^-8 of it at most)."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().float().cpu().double().numpy()


def make(lengths, vocab, dtype, dev, seed, pad=0, lead=0, tail=0, ignore=0.3, offset=0):
    """logits (rows `pad` elements apart, from element `offset` of their buffer), labels, offsets."""
    g = torch.Generator().manual_seed(seed)
    rows = lead + sum(lengths) + tail
    buf = torch.full((rows * (vocab + pad) + offset,), float("nan"))
    x = buf[offset:].view(rows, vocab + pad)
    x[:, :vocab] = torch.randn(rows, vocab, generator=g) * 3.0
    labels = torch.randint(0, vocab, (rows,), generator=g)
    x[torch.arange(rows), labels] += 4.0
    labels[torch.rand(rows, generator=g) < ignore] = -100
    offsets = torch.tensor(np.cumsum([lead] + list(lengths)), dtype=torch.int64)
    flat = buf.to(TYPES[dtype]).to(dev)
    return (flat[offset:].view(rows, vocab + pad)[:, :vocab], labels.to(dev), offsets.to(dev))


def reference(x, labels, offsets, ref, beta, kind, smoothing, margin, average):
    """Everything in 64 bits, and the errors that lse, logp may have."""
    rows, V = x.shape
    top = x.max(1, keepdims=True)
    e = np.exp(x - top)
    s = e.sum(1)
    lse = top[:, 0] + np.log(s)
    err = (V / 256 + 60 + 4) * U + 2 * U * (e * np.abs(x - top)).sum(1) / s
    n = (len(offsets) - 1) // 2
    counted = (labels >= 0) & (np.arange(rows) >= offsets[0]) & (np.arange(rows) < offsets[-1])
    logp = np.where(counted, x[np.arange(rows), np.maximum(labels, 0)] - lse, 0.0)
    sums, errs, counts = [], [], []
    for q in range(2 * n):
        at = slice(offsets[q], offsets[q + 1])
        k = counted[at].sum()
        div = max(k, 1) if average else 1
        sums.append(logp[at].sum() / div)
        errs.append(((err[at] + 2 * U * np.abs(logp[at])) * counted[at]).sum() / div)
        counts.append(div)
    sums, errs, counts = np.array(sums), np.array(errs), np.array(counts)
    gain = sums - (0 if ref is None else ref)
    D = gain[:n] - gain[n:]
    derr = errs[:n] + errs[n:]
    z = beta * D - margin
    if kind == "square":
        losses, slope = (D - 0.5 / beta) ** 2, 2 * (D - 0.5 / beta)
        curve = 2.0 + 0 * D
    elif kind == "hinge":
        losses, slope, curve = np.maximum(0, 1 - z), np.where(z < 1, -beta, 0.0), 0 * z
    else:
        sig = np.exp(-np.logaddexp(0.0, -z))
        losses = (1 - smoothing) * np.logaddexp(0.0, -z) + smoothing * np.logaddexp(0.0, z)
        slope = beta * (sig - (1 - smoothing))
        curve = 0.25 * beta * beta + 0 * z
    dlogp = np.zeros(rows)
    dl_err = np.zeros(rows)
    for q in range(2 * n):
        at = slice(offsets[q], offsets[q + 1])
        sign = 1.0 if q < n else -1.0
        dlogp[at] = np.where(counted[at], sign * slope[q % n] / n / counts[q], 0.0)
        # (sig's own roundings: an absolute 8 u of beta)
        dl_err[at] = (curve[q % n] * derr[q % n] + 8 * U * beta * (kind == "sigmoid")) / n / counts[q]
    return dict(lse=np.where(counted, lse, 0), lse_err=err + U * np.abs(lse), logps=sums,
                logps_err=errs + U * np.abs(sums), losses=losses,
                losses_err=np.abs(slope) * derr + curve * derr ** 2 + 8 * U * (np.abs(losses) + 1),
                dlogp=dlogp, dlogp_err=dl_err, counted=counted)


def check_forward(got, r):
    assert np.all(np.abs(f64(got.logps) - r["logps"]) <= r["logps_err"])
    assert np.all(np.abs(f64(got.losses) - r["losses"]) <= r["losses_err"])
    assert abs(float(got.loss) - r["losses"].mean()) <= r["losses_err"].mean() + 2 * U * abs(r["losses"].mean())
    if got.lse is not None:
        assert np.all(np.abs(f64(got.lse) - r["lse"]) <= r["lse_err"])
        assert np.all(np.abs(f64(got.dlogp) - r["dlogp"]) <= r["dlogp_err"] + 4 * U * np.abs(r["dlogp"]))
        assert np.all(f64(got.lse)[~r["counted"]] == 0) and np.all(f64(got.dlogp)[~r["counted"]] == 0)


def check_gradient(d, x, labels, lse, dlogp, dloss, dtype):
    scale = (dlogp * dloss * (labels >= 0))[:, None]
    with np.errstate(invalid="ignore"):
        p = np.where(scale != 0, np.exp(x - lse[:, None]), 0.0)
    hit = np.arange(x.shape[1])[None] == labels[:, None]
    want = scale * (hit - p)
    dist = np.where(p > 0, np.abs(x - lse[:, None]), 0.0)
    lim = np.abs(scale) * p * (2 * U * dist + 10 * U) + 4 * U * np.abs(want) + 2.0 ** -126
    lim += (2.0 ** -8 if dtype == "bf16" else U) * np.abs(want)
    assert np.all(np.abs(f64(d) - want) <= lim)
    assert np.all(f64(d)[scale[:, 0] == 0] == 0)


# lengths of the sequences, vocabulary, padding of the rows, leading and trailing rows, offset
SHAPES = [
    ([1, 1], 1, 0, 0, 0, 0), ([1, 1], 7, 0, 0, 0, 0), ([3, 2], 33, 3, 1, 2, 1),
    ([0, 4], 130, 0, 0, 0, 0), ([5, 0, 3, 7], 1000, 8, 0, 4, 0), ([4, 4, 4, 4, 4, 4], 2049, 1, 2, 0, 3),
    ([1, 1], 32000, 0, 0, 0, 0), ([2, 3], 50257, 47, 0, 1, 0), ([1, 2], 160001, 0, 0, 0, 0),
    ([40, 25, 33, 61], 4096, 0, 0, 3, 0), ([90] * 8, 520, 0, 0, 0, 0), ([2] * 600, 40, 0, 0, 0, 0),
    ([200, 301], 8200, 8, 0, 0, 8), ([2500, 1300], 24, 0, 0, 0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,smoothing,margin,average", [
    ("sigmoid", 0.0, 0.0, False), ("sigmoid", 0.2, 0.5, True), ("hinge", 0.0, 0.1, False),
    ("square", 0.0, 0.0, True)])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{len(s[0])}x{s[1]}" for s in SHAPES])
def test_both_passes_match_the_formulas(lib, gpu, shape, kind, smoothing, margin, average, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    lengths, vocab, pad, lead, tail, offset = shape
    x, labels, offsets = make(lengths, vocab, dtype, gpu, 3, pad, lead, tail, offset=offset)
    g = torch.Generator().manual_seed(8)
    xs, ls, os_ = f64(x), labels.cpu().numpy(), offsets.cpu().numpy()
    base = reference(xs, ls, os_, None, 0.3, kind, smoothing, margin, average)
    ref = torch.tensor(base["logps"]).float() + torch.randn(len(lengths), generator=g)
    got = fo.preference_loss(x, labels, offsets, ref.to(gpu), 0.3, kind, smoothing, margin, average)
    r = reference(xs, ls, os_, ref.double().numpy(), float(np.float32(0.3)), kind,
                  float(np.float32(smoothing)), float(np.float32(margin)), average)
    check_forward(got, r)
    dloss = torch.tensor(1.7, device=gpu)
    d = fo.preference_loss_backward(x, labels, got.lse, got.dlogp, dloss)
    check_gradient(d, xs, ls, f64(got.lse), f64(got.dlogp), f64(dloss), dtype)
    # an output at another position within 16 bytes takes the other path
    n = vocab + 5
    buf = torch.full((x.shape[0] * n + 1,), float("nan"), dtype=x.dtype, device=gpu)
    other = buf[1:].view(-1, n)[:, :vocab]
    fo.preference_loss_backward(x, labels, got.lse, got.dlogp, dloss, out=other)
    assert torch.equal(other, d)
    assert torch.isnan(buf[1:].view(-1, n)[:, vocab:]).all() and torch.isnan(buf[0])
    # in place
    assert fo.preference_loss_backward(x, labels, got.lse, got.dlogp, dloss, out=x) is x
    assert torch.equal(x, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_uncounted_rows_may_hold_anything_and_masked_logits_count_for_nothing(lib, gpu, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    lowest = torch.finfo(TYPES[dtype]).min
    for vocab in (300, 20000):
        x, labels, offsets = make([6, 5], vocab, dtype, gpu, 4, tail=2, ignore=0.0)
        labels[2] = -1
        x[2] = float("nan")
        x[11], x[12] = float("inf"), float("nan")          # behind the last sequence
        x[0, 5:40] = float("-inf")
        x[1, 5:40] = lowest
        x[4] = lowest                                       # all of it: an even distribution
        labels[0], labels[1], labels[4] = 3, 2, 7
        got = fo.preference_loss(x, labels, offsets)
        xs, ls = f64(x), labels.cpu().numpy()
        xs[2] = xs[11] = xs[12] = 0.0
        # (the formulas in 64 bits, with -1e30 for -inf; a row of the lowest value as one of 0)
        xs[4] = 0.0
        xs[0, 5:40] = xs[1, 5:40] = -1e30
        r = reference(xs, ls, offsets.cpu().numpy(), None, float(np.float32(0.1)), "sigmoid", 0, 0, False)
        lse = f64(got.lse)
        assert lse[4] == pytest.approx(lowest) and lse[2] == lse[11] == lse[12] == 0
        lse[4] = r["lse"][4]
        for name in ("logps", "losses"):
            assert np.all(np.abs(f64(getattr(got, name)) - r[name]) <= r[name + "_err"])
        assert np.all(np.abs(lse - r["lse"])[[0, 1, 3]] <= r["lse_err"][[0, 1, 3]])
        d = fo.preference_loss_backward(x, labels, got.lse, got.dlogp)
        assert torch.isfinite(d).all()
        assert (d[0, 5:40] == 0).all() and (d[1, 5:40] == 0).all()
        assert (d[2] == 0).all() and (d[11:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_rows_and_labels_past_the_vocabulary_are_seen(lib, gpu, dtype):
    from paper_2608_15665_gb300 import firstorder as fo
    for vocab in (300, 20000):
        for spoil in ("nan", "inf", "empty", "label"):
            x, labels, offsets = make([3, 3, 3, 3], vocab, dtype, gpu, 5, ignore=0.0)
            if spoil == "nan":
                x[1, 17] = float("nan")
            elif spoil == "inf":
                x[1, 17] = float("inf")
            elif spoil == "empty":
                x[1] = float("-inf")
            else:
                labels[1] = vocab
            got = fo.preference_loss(x, labels, offsets)
            assert torch.isnan(got.logps).tolist() == [True, False, False, False]
            assert torch.isnan(got.losses).tolist() == [True, False] and torch.isnan(got.loss)


def test_offsets_out_of_range_touch_nothing_outside(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    x, labels, _ = make([3, 3], 50, "f32", gpu, 6)
    for offsets in ([0, 3, 100], [-5, 3, 6], [5, 2, 6], [0, 2 ** 62, 2 ** 62 + 5], [4, 4, 4],
                    [-2 ** 62, -2 ** 61, 2 ** 62]):
        got = fo.preference_loss(x, labels, torch.tensor(offsets, device=gpu))
        fo.preference_loss_backward(x, labels, got.lse, got.dlogp)
    torch.cuda.synchronize()


def test_no_rows(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    x = torch.zeros(0, 10, device=gpu)
    got = fo.preference_loss(x, torch.zeros(0, dtype=torch.int64, device=gpu),
                             torch.zeros(5, dtype=torch.int64, device=gpu), torch.ones(4, device=gpu))
    assert float(got.loss) == pytest.approx(np.log(2.0), rel=1e-6)
    assert (got.logps == 0).all() and got.lse.shape == (0,)
    assert fo.preference_loss_backward(x, torch.zeros(0, dtype=torch.int64, device=gpu), got.lse,
                                       got.dlogp).shape == (0, 10)


@pytest.mark.parametrize("z", [0.0, 1.0, -30.0, 40.0, 200.0, -200.0])
def test_far_pairs(lib, gpu, z):
    """The loss and its slope where one side saturates, by the reference's share alone."""
    from paper_2608_15665_gb300 import firstorder as fo
    x, labels, offsets = make([2, 2], 64, "f32", gpu, 7, ignore=1.0)
    labels.fill_(-1)
    labels[0], labels[2] = 1, 1
    x[2] = x[0]
    ref = torch.tensor([-z / 0.5, 0.0], device=gpu)
    got = fo.preference_loss(x, labels, offsets, ref, beta=0.5)
    want = np.logaddexp(0.0, -z)
    assert float(got.loss) == pytest.approx(want, rel=1e-5, abs=1e-38)
    slope = -0.5 * np.exp(-np.logaddexp(0.0, z))
    assert float(got.dlogp[0]) == pytest.approx(slope, rel=1e-5, abs=1e-38)
    assert float(got.dlogp[2]) == -float(got.dlogp[0])


def test_gradient_is_the_difference_quotient_and_autograd_takes_it(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    x, labels, offsets = make([4, 3, 5, 6], 90, "f32", gpu, 9)
    leaf = x.clone().requires_grad_()
    loss = fo.PreferenceLoss.apply(leaf, labels, offsets, None, 0.4, "sigmoid", 0.1, 0.2, False)
    (2.0 * loss).backward()
    g = torch.Generator().manual_seed(2)
    v = torch.randn(x.shape, generator=g).to(gpu)
    os_, ls = offsets.cpu().numpy(), labels.cpu().numpy()

    def at(h):
        r = reference(f64(x) + h * f64(v), ls, os_, None, float(np.float32(0.4)), "sigmoid",
                      float(np.float32(0.1)), float(np.float32(0.2)), False)
        return 2.0 * r["losses"].mean()
    h = 1e-4
    quotient = (at(h) - at(-h)) / (2 * h)
    assert float((leaf.grad * v).double().sum()) == pytest.approx(quotient, rel=1e-4)
    with pytest.raises(RuntimeError):
        twice, = torch.autograd.grad(fo.PreferenceLoss.apply(leaf, labels, offsets), leaf,
                                     create_graph=True)
        twice.sum().backward()
    # bf16, and no gradient asked for
    with torch.no_grad():
        fo.PreferenceLoss.apply(x.bfloat16(), labels, offsets)


def test_capture_replay_and_other_streams(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    x, labels, offsets = make([30, 20, 25, 41], 3000, "bf16", gpu, 10)
    y, _, _ = make([30, 20, 25, 41], 3000, "bf16", gpu, 11)
    want = []
    for data in (x, y):
        got = fo.preference_loss(data, labels, offsets)
        want.append((got.loss.clone(), fo.preference_loss_backward(data, labels, got.lse, got.dlogp)))
    buf = x.clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = fo.preference_loss(buf, labels, offsets)
        d = fo.preference_loss_backward(buf, labels, got.lse, got.dlogp)
    for data, (loss, grad) in zip((y, x), reversed(want)):
        buf.copy_(data)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got.loss, loss) and torch.equal(d, grad)
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        buf.copy_(y)
        got = fo.preference_loss(buf, labels, offsets)
    s.synchronize()
    assert torch.equal(got.loss, want[1][0])


def test_a_loss_is_a_place_in_a_subspace_steps_losses(lib, gpu):
    """SubZeroPlus steps by losses that never come to the host, and by their values."""
    from paper_2608_15665_gb300 import firstorder as fo
    from paper_2608_15665_gb300.schedule import SubZeroPlus
    x, labels, offsets = make([12, 9, 11, 10], 256, "bf16", gpu, 12)
    g = torch.Generator().manual_seed(1)
    start = (torch.randn(256, 128, generator=g) * 0.05).to(torch.bfloat16)
    X = torch.randn(x.shape[0], 128, generator=g).to(torch.bfloat16).to(gpu)
    out = []
    for on_device in (True, False):
        W = start.clone().to(gpu)
        z = SubZeroPlus([W], 16, 2, seed=5)
        z.init_subspace(0)

        def loss_fn(t, index):
            loss = fo.preference_loss(z.linear_perturbed(0, X), labels, offsets, grad=False).loss
            return loss if on_device else float(loss)
        for t in range(3):
            z.run_step_linear(t, t + 1, loss_fn, "central", 1e-2, 1e-2, 0.9, 0.95, 1e-8)
        z.sync()
        out.append(W)
        z.close()
    assert torch.equal(*out) and not torch.equal(out[0].cpu(), start)
    slots = torch.zeros(3, device=gpu)
    got = fo.preference_loss(x, labels, offsets, out=slots[1:2])
    assert float(slots[1]) == float(got.losses.mean()) or abs(float(slots[1] - got.losses.mean())) < 1e-6
    assert float(slots[0]) == float(slots[2]) == 0.0
