"""Hybrid fine-tuning of a small model: the body by subspace zeroth-order steps, the tail by
backpropagation.

    python examples/hybrid_tail.py [steps]

The body is a residual stack of linear layers and norms.  Its matrices are never
differentiated: SubZeroPlus evaluates the loss at perturbed weights inside the forward GEMMs
and applies the orthogonalised subspace moment (ZO_OPT_MUON).  The tail -- the last norm and
the classifier -- costs one backward pass through itself alone and no activations of the
body: the norm's weight and bias take their gradients from layer_norm_backward, the
classifier's matrix the Muon step on its full gradient.

Synthetic tokens whose labels come from a random teacher.
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_15665_gb300 import binding as zb                      # noqa: E402
from paper_2608_15665_gb300 import firstorder as fo                   # noqa: E402
from paper_2608_15665_gb300.schedule import SubZeroPlus               # noqa: E402

HIDDEN, LAYERS, CLASSES, TOKENS = 256, 2, 32, 512
RANK, QUERIES, EPS = 16, 4, 1e-2


class Model:
    def __init__(self, device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, scale=1.0):
            return (torch.randn(*shape, generator=g) * scale).to(torch.bfloat16).to(device)

        self.x = normal(TOKENS, HIDDEN)
        teacher = normal(HIDDEN, CLASSES)
        self.labels = (self.x.float() @ teacher.float()).argmax(1)
        # body: W_i of every block, and the parameters of the norm in front of it
        self.body = [normal(HIDDEN, HIDDEN, scale=HIDDEN ** -0.5) for _ in range(LAYERS)]
        self.ones = torch.ones(HIDDEN, device=device)
        self.zeros = torch.zeros(HIDDEN, device=device)
        # tail: norm (fp32) and classifier (bf16)
        self.weight, self.bias = self.ones.clone(), self.zeros.clone()
        self.head = normal(CLASSES, HIDDEN, scale=0.02)
        self.head_grad = torch.zeros_like(self.head)
        self.zo = SubZeroPlus(self.body, RANK, QUERIES, seed=7)
        self.zo.init_subspace(0)
        self.muon = fo.Muon([self.head], [self.head_grad])

    def body_forward(self):
        """The tail's input, at the body's prepared evaluation point."""
        h, branch = self.x, None
        for i in range(LAYERS):
            out = fo.layer_norm(h, self.ones, self.zeros, residual=branch, stats=False)
            h = out.h if branch is not None else h
            branch = torch.relu(self.zo.linear_perturbed(i, out.y))
        return h, branch

    def loss(self, h, branch):
        out = fo.layer_norm(h, self.weight, self.bias, residual=branch)
        logits = out.y.float() @ self.head.float().t()
        return torch.nn.functional.cross_entropy(logits, self.labels), logits, out

    def tail_step(self, lr_norm, lr_head):
        """One backward pass through the tail, at the body's present weights."""
        self.zo.linear_prepare(0, 0, 0.0, eps=EPS)                    # C = 0: W itself
        loss, logits, out = self.loss(*self.body_forward())
        p = torch.softmax(logits, 1)
        p[torch.arange(TOKENS, device=p.device), self.labels] -= 1.0
        dlogits = p / TOKENS
        self.head_grad.copy_(dlogits.t() @ out.y.float())
        dy = (dlogits @ self.head.float()).to(torch.bfloat16)
        _, dweight, dbias = fo.layer_norm_backward(dy, out.h, self.weight, out.mean, out.rstd)
        self.weight.sub_(dweight, alpha=lr_norm)
        self.bias.sub_(dbias, alpha=lr_norm)
        self.muon.step(lr=lr_head, momentum=0.9)
        return float(loss)

    def body_step(self, t, lr):
        """One subspace step of the body: losses at W +- eps U Z V^T, forward passes only."""
        def loss_fn(_t, _index):
            return float(self.loss(*self.body_forward())[0])
        self.zo.run_step_linear(t, t + 1, loss_fn, "central", EPS, lr, 0.9, 0.0, 1e-8,
                                optimizer=zb.ZO_OPT_MUON)

    def close(self):
        self.zo.close()
        self.muon.close()


def train(steps=40, lr_body=0.02, lr_norm=0.5, lr_head=0.02, device="cuda"):
    """Losses before each step."""
    model = Model(device)
    losses = []
    for t in range(steps):
        losses.append(model.tail_step(lr_norm, lr_head))
        model.body_step(t, lr_body)
    losses.append(float(model.tail_step(0.0, 0.0)))
    model.zo.sync()
    model.muon.sync()
    fo.layer_norm_sync()
    model.close()
    return losses


if __name__ == "__main__":
    curve = train(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
    for step in range(0, len(curve), max(1, len(curve) // 10)):
        print(f"step {step:3d}  loss {curve[step]:.4f}")
    print(f"last       loss {curve[-1]:.4f}")
