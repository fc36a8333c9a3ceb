"""How many 8-bit codes of AdamW's steps the 64-bit formulas leave open: in no tensor and neither
state more than one element or one in a hundred.

An element is open where its value in steps, plus its random part, is nearer to a whole number than the
errors of an fp32 evaluation: 3 u of m's sum of magnitudes and 6 u of r in steps (u = 2^-24; at most 16
steps to a value, more where m cancels), and 2^-19: twice that of an interval of 1.  With m's terms ten
times as large as m itself that is 2 (16 x 30 u + 2^-19) = 6e-5 of all elements: 0.25 of 4096, one of
all with a chance of 1 in 4, and a hundredth is 160 times as much."""

import pytest
import torch

from test_gpu_adamw import B1, B2, EPS, LR, SHAPES, U, WD, check_codes, f64, make, random_of, values

import numpy as np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,gdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_codes_are_pinned_in_every_tensor(lib, gpu, dtype, gdtype):
    from paper_2608_15665_gb300 import firstorder as fo
    W, G = (list(t) for t in zip(*[make(s, dtype, gdtype, gpu, i, offset=i % 2) for i, s in enumerate(SHAPES)]))
    seed = (1 << 40) + 6
    opt = fo.AdamW(W, G, bits=8, seed=seed)
    for t in range(1, 4):
        before = [(f64(x), values(s.m, s.m_exp, w.shape), values(s.v, s.v_exp, w.shape) ** 2)
                  for w, x, s in zip(W, G, opt.states)]
        opt.step(LR, (B1, B2), EPS, WD)
        torch.cuda.synchronize()
        for i, (w, s, (x, m, v)) in enumerate(zip(W, opt.states, before)):
            m1, root = (B1 * m + (1 - B1) * x).reshape(-1), np.sqrt(B2 * v + (1 - B2) * x * x).reshape(-1)
            size = (B1 * np.abs(m) + (1 - B1) * np.abs(x)).reshape(-1)
            r = random_of(seed, i, t, w.numel())
            few = max(1.0 / w.numel(), 0.01) * (1 + 1e-9)
            assert check_codes(s.m, s.m_exp, m1, np.abs(m1), r, 3 * U * size, False) <= few, (t, i)
            assert check_codes(s.v, s.v_exp, root, root, r, 6 * U * root, True) <= few, (t, i)
        for k, x in enumerate(G):
            x.mul_(-0.7 if k % 2 else 1.6)
    opt.close()
