"""The waits of the orthogonalisation's product kernel, read from its source (no GPU needed).

A bounded wait gives each lane its own answer: lanes start their clocks apart, so of a warp some
may see the limit pass and some the barrier.  Warp-wide instructions follow every wait of this
kernel, so what a warp does next has to go by one answer for all lanes, and lane 0, which
reports a wait that ran out, has to have it too.  ``warp_wait`` gives that answer; a plain wait
may stand only where nothing depends on what it returns."""

import os
import re

from conftest import ROOT

SOURCE = os.path.join(ROOT, "paper_2608_15665_gb300", "csrc", "zo_ortho_gemm.cu")


def _statements(text):
    """(statement up to the wait, the enclosing code before it) of every bounded wait."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"\bmbar_wait_bounded\s*\(", text):
        start = max(text.rfind(c, 0, m.start()) for c in ";{}\n")
        yield text[start + 1:m.start()].strip()


def test_no_lane_goes_by_a_wait_of_its_own():
    with open(SOURCE) as f:
        text = f.read()
    whole = [s for s in _statements(text) if not s.startswith("return __all_sync(")]
    assert len(whole) + 1 == len(list(_statements(text)))        # warp_wait is there, once
    # what is left waits for copies or MMAs before the kernel ends: a call on its own, at most
    # under a condition that does not go by a wait
    for s in whole:
        assert re.fullmatch(r"(if \([^()]*\))?", s), s


def test_waits_are_by_converged_warps():
    """A lane that requested boxes joins its warp again before the warp's next wait."""
    with open(SOURCE) as f:
        text = f.read()
    body = text[text.index("int64_t n_acc = 0;"):]
    loop = body[body.index("request(q);"):]
    before_wait = loop[:loop.index("_wait")]
    assert "__syncwarp()" in before_wait
