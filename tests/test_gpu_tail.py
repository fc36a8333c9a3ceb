"""A model's tail as its user runs it: norm, gated linear block, norm, head, preference loss, one
backward pass through them, and AdamW and Muon steps on the gradients -- against the same tail in
64 bits with torch's own differentiation."""

import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
D, F, V = 128, 264, 520
LENGTHS = [9, 14, 11, 6]


class Tail:
    def __init__(self, dev, seed=0):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, scale=1.0):
            return (torch.randn(*shape, generator=g) * scale).to(BF).to(dev)
        rows = sum(LENGTHS)
        self.x = normal(rows, D)
        self.params = dict(n1=torch.ones(D, device=dev), b1=torch.zeros(D, device=dev),
                           wg=normal(F, D, scale=D ** -0.5), wu=normal(F, D, scale=D ** -0.5),
                           down=normal(D, F, scale=F ** -0.5), n2=torch.ones(D, device=dev),
                           b2=torch.zeros(D, device=dev), head=normal(V, D, scale=2 * D ** -0.5))
        self.labels = torch.randint(0, V, (rows,), generator=g).to(dev)
        self.labels[::5] = -100
        ends = torch.tensor([0] + LENGTHS).cumsum(0)
        self.offsets = ends.to(dev)

    def loss(self, p):
        """bf16 activations, the framework's operators."""
        from paper_2608_15665_gb300 import firstorder as fo
        h = fo.LayerNorm.apply(self.x, p["n1"], p["b1"], 1e-5)
        h = fo.GatedLinear.apply(h, p["wg"], p["wu"], "silu")
        h = fo.LayerNorm.apply(self.x + h @ p["down"].t(), p["n2"], p["b2"], 1e-5)
        return fo.PreferenceLoss.apply(h @ p["head"].t(), self.labels, self.offsets, None, 0.2)

    def loss64(self, p):
        x = self.x.double()
        ln = torch.nn.functional.layer_norm
        h = ln(x, (D,), p["n1"], p["b1"], 1e-5)
        h = torch.nn.functional.silu(h @ p["wg"].t()) * (h @ p["wu"].t())
        h = ln(x + h @ p["down"].t(), (D,), p["n2"], p["b2"], 1e-5)
        logp = torch.log_softmax(h @ p["head"].t(), 1)
        logp = logp.gather(1, self.labels.clamp(min=0)[:, None])[:, 0] * (self.labels >= 0)
        s = [part.sum() for part in logp.split(LENGTHS)]
        z = [0.2 * (s[k] - s[k + 2]) for k in range(2)]
        return -torch.nn.functional.logsigmoid(torch.stack(z)).mean()


def test_gradients_of_a_tail(lib, gpu):
    from paper_2608_15665_gb300 import firstorder as fo
    tail = Tail(gpu)
    leaves = {k: v.clone().requires_grad_() for k, v in tail.params.items()}
    wide = {k: v.double().requires_grad_() for k, v in tail.params.items()}
    loss = tail.loss(leaves)
    loss.backward()
    want = tail.loss64(wide)
    want.backward()
    # activations are rounded to bf16 (2^-9) five times on the way to logits of size ~2 and to sums
    # of ~8 of them: z is off by at most 0.2 x 16 rows x 2 x 5 x 2^-9
    assert abs(float(loss.detach()) - float(want.detach())) <= 0.2 * 16 * 2 * 5 * 2.0 ** -9
    for k, leaf in leaves.items():
        g, w = leaf.grad.double(), wide[k].grad
        # a dozen roundings of 2^-9 on the way down and back, in random directions
        assert float((g - w).norm()) <= 12 * 2.0 ** -9 * float(w.norm()), k
    fo.layer_norm_sync()
    fo.gated_linear_sync()


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_of_a_tail_follow_64_bits(lib, gpu, bits):
    """Three steps: AdamW on norms, down projection and head, Muon on the gated block's matrices; the
    tail's loss and parameters against AdamW in 64 bits from the same gradients."""
    from paper_2608_15665_gb300 import firstorder as fo
    tail = Tail(gpu)
    p = {k: v.clone().requires_grad_() for k, v in tail.params.items()}
    names = [k for k in p if k not in ("wg", "wu")]
    with torch.no_grad():
        muon = fo.Muon([p["wg"].detach(), p["wu"].detach()])
        adamw = fo.AdamW([p[k].detach() for k in names], [torch.zeros_like(p[k]) for k in names],
                         bits=bits, seed=1)
    m = {k: torch.zeros(p[k].shape, dtype=torch.float64, device=gpu) for k in names}
    v = {k: torch.zeros_like(t) for k, t in m.items()}
    losses = []
    for t in range(1, 4):
        loss = tail.loss(p)
        losses.append(float(loss.detach()))
        grads = dict(zip(p, torch.autograd.grad(loss, list(p.values()))))
        before = {k: p[k].detach().double().clone() for k in names}
        for k, buf in zip(names, adamw.grads):
            buf.copy_(grads[k])
        for k, buf in zip(("wg", "wu"), muon.grads):
            buf.copy_(grads[k])
        adamw.step(lr=1e-3, weight_decay=0.01)
        muon.step(lr=1e-3)
        for i, k in enumerate(names):
            g = grads[k].double()
            m[k] = 0.9 * m[k] + 0.1 * g
            v[k] = 0.999 * v[k] + 0.001 * g * g
            step = 1e-3 * (m[k] / (1 - 0.9 ** t)) / ((v[k] / (1 - 0.999 ** t)).sqrt() + 1e-8)
            want = before[k] * (1 - 1e-5) - step
            off = (p[k].detach().double() - want).abs()
            # a rounding, W's two in fp32, and 28 of 2^-24 of an update of at most three steps
            lim = (2.0 ** -8 if p[k].dtype == BF else 2.0 ** -22) * want.abs() + 1e-3 * 2.0 ** -15
            assert float((off - lim).max()) <= 0, (k, t)
            if bits == 8:                                  # go on from the codes' values
                s = adamw.states[i]
                for mean, code, e, power in ((m, s.m, s.m_exp, 1), (v, s.v, s.v_exp, 2)):
                    scale = 2.0 ** (e.double().clamp(min=40) - 134)
                    wide = code.double() * scale.repeat_interleave(256)[:code.numel()]
                    mean[k] = (wide ** power).view(g.shape)
    adamw.close()
    muon.sync()
    muon.close()
    assert all(l == l for l in losses)


def test_calls_at_once_on_two_streams(lib, gpu):
    """Blocks, losses and AdamW handles on two streams at the same time: the bits of calls alone."""
    from paper_2608_15665_gb300 import firstorder as fo
    g = torch.Generator().manual_seed(3)
    x = [torch.randn(t, 128, generator=g).to(BF).to(gpu) for t in (100, 700)]
    wg, wu = (torch.randn(1032, 128, generator=g).mul_(0.1).to(BF).to(gpu) for _ in range(2))
    logits = [torch.randn(40, v, generator=g).to(gpu) for v in (900, 33000)]
    labels = torch.randint(0, 900, (40,), generator=g).to(gpu)
    offsets = torch.tensor([0, 9, 23, 34, 40], device=gpu)

    def work(k, handle):
        out = fo.gated_linear(x[k], wg, wu, save=True)
        grads = fo.gated_linear_backward(out.h, x[k], wg, wu, out.gate, out.up)
        got = fo.preference_loss(logits[k], labels, offsets)
        d = fo.preference_loss_backward(logits[k], labels, got.lse, got.dlogp)
        handle.step(lr=1e-2)
        return [out.h, *grads, got.loss, got.logps, d]

    def handles():
        out = []
        for k in range(2):
            W = torch.arange(50000, device=gpu, dtype=torch.float32) * 1e-5 * (k + 1)
            out.append(fo.AdamW([W], [torch.sin(W)], bits=8, seed=k))
        torch.cuda.synchronize()
        return out
    alone = handles()
    want = [work(k, alone[k]) for k in range(2)]
    for _ in range(3):
        for h in alone:
            h.step(lr=1e-2)
    torch.cuda.synchronize()
    pair = handles()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(4):
        for k, s in enumerate(streams):
            s.wait_stream(torch.cuda.default_stream())
            with torch.cuda.stream(s):
                got[k] = work(k, pair[k])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[k], want[k]))
        assert torch.equal(pair[k].weights[0], alone[k].weights[0])
    fo.gated_linear_sync()
