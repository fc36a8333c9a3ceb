"""The hybrid example: subspace steps below, backpropagation of the tail, the same optimiser
in both.  512 tokens with 256 features are linearly separable into their 32 classes, and a
Muon step of 0.02 moves a logit by up to 0.02 |y| = 0.3, so forty steps take the loss well
below its start at ln 32 = 3.47; a third less is asked for."""

import importlib.util
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def test_the_loss_falls(lib, gpu):
    spec = importlib.util.spec_from_file_location("hybrid_tail",
                                                  os.path.join(ROOT, "examples", "hybrid_tail.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(40)
    assert all(x == x and x < 10.0 for x in losses)
    assert losses[-1] < 2.0 * losses[0] / 3.0
