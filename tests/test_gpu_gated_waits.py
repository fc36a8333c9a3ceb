"""The gated linear block when waits inside its kernels run out: every element of a result is right bit
for bit or NaN, and the status says so once.  Libraries built from the same sources report such
waits on request; copies and products go on as ever, and the last waits, for what is in flight, are the
real ones."""

import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from test_gpu_gated import BF, inputs, make

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("zo_gated_forward", "zo_gated_backward", "zo_gated_sync_status")


@pytest.fixture(scope="module")
def probe(lib, gpu, tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    so = str(tmp_path_factory.mktemp("probe") / "probe.so")
    csrc, harness = (os.path.join(ROOT, *p) for p in (("paper_2608_15665_gb300", "csrc"), ("tests", "harness")))
    subprocess.run([nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-O3", "-std=c++17", "-shared",
                    "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr", "-I", csrc, "-I", harness,
                    os.path.join(harness, "gated_wait_probe_gemm.cu"),
                    os.path.join(harness, "gated_wait_probe_few.cu"), os.path.join(csrc, "zo_gated.cu"),
                    "-o", so], check=True, capture_output=True, text=True)
    loaded = ctypes.CDLL(so)
    for name in NAMES:
        fn = getattr(loaded, name)
        fn.restype, fn.argtypes = lib._SIGNATURES[name]
    for name in ("probe_plan", "probe_parts"):
        getattr(loaded, name).argtypes = [ctypes.c_longlong] * 3
    return loaded


# tokens, D, F: few tokens, with K in one round of the stages and in several; tiles of tokens in few and
# many rounds; turned ones with two accumulators and with one; dX's K whole and in parts, and with two
# rows a token
SHAPES = [(3, 64, 200), (40, 4096, 304), (128, 264, 2000), (256, 512, 5632), (2304, 256, 2064),
          (1100, 512, 5504), (777, 5120, 13824), (2304, 4096, 1032)]


def _forward(L, lib, x, wg, wu, out):
    (T, D), F = x.shape, wg.shape[0]
    h, g, u = (t.data_ptr() for t in out)
    return L.zo_gated_forward(x.data_ptr(), D, T, D, wg.data_ptr(), D, wu.data_ptr(), D, F, lib.ZO_GATED_SILU,
                              h, F, g, F, u, F, None)


def _backward(L, lib, dh, x, wg, wu, g, u, out, ws):
    (T, D), F = x.shape, wg.shape[0]
    dx, dwg, dwu = (t.data_ptr() for t in out)
    return L.zo_gated_backward(dh.data_ptr(), F, x.data_ptr(), D, T, D, wg.data_ptr(), D, wu.data_ptr(), D, F,
                               lib.ZO_GATED_SILU, g.data_ptr(), F, u.data_ptr(), F, dx, D, dwg, D, dwu, D,
                               ws.data_ptr(), ws.numel(), None)


def _fresh(like):
    return [torch.full_like(t, 7.0) for t in like]


def _nan_count(got, want):
    """How many are NaN; all others have to be right."""
    n = 0
    for a, b in zip(got, want):
        nan = torch.isnan(a)
        assert bool(((a == b) | nan).all())
        n += int(nan.sum())
    return n


@pytest.mark.parametrize("T,D,F", SHAPES, ids=[f"{t}x{d}x{f}" for t, d, f in SHAPES])
def test_results_whose_sums_were_not_waited_for(lib, gpu, probe, T, D, F):
    x, wg, wu = inputs(T, D, F, gpu)
    dh = make(T, F, gpu, 4, 0.1)
    ws = torch.empty(lib.zo_gated_workspace(T, D, F), dtype=torch.uint8, device=gpu)
    fwd = [torch.empty(T, F, dtype=BF, device=gpu) for _ in range(3)]
    bwd = [torch.empty(s, dtype=BF, device=gpu) for s in ((T, D), (F, D), (F, D))]
    assert _forward(lib.LIB, lib, x, wg, wu, fwd) == 0
    assert _backward(lib.LIB, lib, dh, x, wg, wu, fwd[1], fwd[2], bwd, ws) == 0
    lib.zo_gated_sync_status()
    lost = set()
    for mode in (0, 1, 2, 3, 4, 5, 6, 7, 8, 0):
        assert probe.probe_lose_gemm(mode) == 0 and probe.probe_lose_few(mode) == 0
        ws.fill_(0xFF)                                      # NaN, and no count of parts
        for want, call in ((fwd, lambda out: _forward(probe, lib, x, wg, wu, out)),
                           (bwd, lambda out: _backward(probe, lib, dh, x, wg, wu, fwd[1], fwd[2], out, ws))):
            got = _fresh(want)
            assert call(got) == 0
            told = probe.zo_gated_sync_status(None)
            assert probe.zo_gated_sync_status(None) == lib.ZO_OK
            n = _nan_count(got, want)
            assert told == lib.ZO_ERR_TIMEOUT or (told == lib.ZO_OK and n == 0), mode
            if mode == 0:
                assert told == lib.ZO_OK
            if mode == 1:
                assert n == sum(t.numel() for t in want)
            if n:
                lost.add((mode, want is fwd))
    # each kind of wait was lost somewhere in the larger shapes
    if T == 2304:
        assert {m for m, _ in lost} >= {1, 2, 3, 4, 5, 6, 7}
    if (T, D) == (40, 4096):
        assert {(m, True) for m in (1, 2, 3, 8)} <= lost
    lib.zo_gated_sync_status()


def test_the_shapes_take_every_kind_of_tile(lib, gpu, probe):
    plans = [probe.probe_plan(*s) for s in SHAPES if s[0] > 128]
    assert any(p > 0 for p in plans) and any(-128 <= p < 0 for p in plans) and any(p < -128 for p in plans)
    parts = [probe.probe_parts(*s) for s in SHAPES]
    assert any(p > 1 for p in parts) and any(p == 1 for p in parts)
