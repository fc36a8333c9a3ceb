"""The losses of a tail that AdamW and Muon steps move, against the same tail in 64 bits at the same
parameters."""

import pytest
import torch

from test_gpu_tail import Tail

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_losses_of_a_tail_that_is_trained(lib, gpu, bits):
    from paper_2608_15665_gb300 import firstorder as fo
    tail = Tail(gpu, seed=1)
    p = {k: v.clone().requires_grad_() for k, v in tail.params.items()}
    names = [k for k in p if k not in ("wg", "wu")]
    muon = fo.Muon([p["wg"].detach(), p["wu"].detach()])
    adamw = fo.AdamW([p[k].detach() for k in names], [torch.zeros_like(p[k]) for k in names], bits=bits)
    for t in range(5):
        loss = tail.loss(p)
        grads = dict(zip(p, torch.autograd.grad(loss, list(p.values()))))
        with torch.no_grad():
            want = float(tail.loss64({k: v.double() for k, v in p.items()}))
        # five roundings to bf16 on the way to logits of size ~2, in sums of ~8 of them
        assert abs(float(loss.detach()) - want) <= 0.2 * 16 * 2 * 5 * 2.0 ** -9
        for handle, keys in ((adamw, names), (muon, ("wg", "wu"))):
            for k, buf in zip(keys, handle.grads):
                buf.copy_(grads[k])
        adamw.step(lr=1e-3, weight_decay=0.01)
        muon.step(lr=1e-3)
    adamw.close()
    muon.sync()
    muon.close()
    fo.layer_norm_sync()
    fo.gated_linear_sync()
