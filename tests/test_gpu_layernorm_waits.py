"""Layer norm when waits for its rows run out: no wrong value is written.  A row of y, of dx and of
the statistics is right bit for bit or NaN throughout, an element of the column sums (and of the
residual's sum) right or NaN, and the status says so once.  A library built from the same sources
reports such waits on request; nothing waits in earnest, and no copy is lost."""

import ctypes
import os
import shutil
import subprocess

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("zo_layernorm_forward", "zo_layernorm_backward", "zo_layernorm_sync_status")


@pytest.fixture(scope="module")
def probe(lib, gpu, tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    so = str(tmp_path_factory.mktemp("probe") / "probe.so")
    subprocess.run([nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-O3", "-std=c++17", "-shared",
                    "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
                    "-I", os.path.join(ROOT, "paper_2608_15665_gb300", "csrc"),
                    os.path.join(ROOT, "tests", "harness", "layernorm_wait_probe.cu"), "-o", so],
                   check=True, capture_output=True, text=True)
    loaded = ctypes.CDLL(so)
    for name in NAMES:
        fn = getattr(loaded, name)
        fn.restype, fn.argtypes = lib._SIGNATURES[name]
    loaded.probe_lose.argtypes = [ctypes.c_int]
    return loaded


# rows, columns, padding: both ways a group of threads makes up a row, on and off 16 bytes, and
# the rings of different depths
SHAPES = [(1900, 1003, 1), (2500, 640, 0), (900, 2048, 8), (700, 2051, 0), (400, 5120, 0),
          (340, 9001, 2), (16000, 1003, 1), (9000, 2048, 0), (1500, 9001, 1)]


def _outputs(x, w):
    return ([torch.full(x.shape, 7.0, dtype=x.dtype, device=x.device) for _ in range(3)]
            + [torch.full((x.shape[0],), 7.0, device=x.device) for _ in range(2)]
            + [torch.full_like(w, 7.0) for _ in range(2)])


def _forward(L, lib, code, x, w, b, r, y, h, mean, rstd):
    rows, n = x.shape
    return L.zo_layernorm_forward(x.data_ptr(), x.stride(0), r.data_ptr() if r is not None else None, n,
                                  rows, n, code, w.data_ptr(), b.data_ptr(), lib.ZO_F32, 1e-5,
                                  y.data_ptr(), n, h.data_ptr() if r is not None else None, n,
                                  mean.data_ptr(), rstd.data_ptr(), None)


def _backward(L, lib, code, dy, x, w, mean, rstd, dr, dx, dw, db, ws):
    rows, n = x.shape
    return L.zo_layernorm_backward(dy.data_ptr(), n, x.data_ptr(), x.stride(0),
                                   dr.data_ptr() if dr is not None else None, n, rows, n, code,
                                   w.data_ptr(), lib.ZO_F32, mean.data_ptr(), rstd.data_ptr(),
                                   dx.data_ptr(), n, dw.data_ptr(), db.data_ptr(), ws.data_ptr(),
                                   ws.numel(), None)


def _right_or_nan(got, want, by_rows):
    same, nan = got == want, torch.isnan(got)
    if by_rows and got.dim() == 2:
        return bool((same.all(1) | nan.all(1)).all())
    return bool((same | nan).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,cols,pad", SHAPES, ids=[f"{s[0]}x{s[1]}" for s in SHAPES])
def test_rows_that_did_not_come_in_time(lib, gpu, probe, rows, cols, pad, residual, dtype):
    g = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, cols + pad, generator=g).to(dtype).to(gpu)[:, :cols]
    dy, r, dr = (torch.randn(rows, cols, generator=g).to(dtype).to(gpu) for _ in range(3))
    w, b = (torch.randn(cols, generator=g).to(gpu) for _ in range(2))
    code = lib.ZO_BF16 if dtype == torch.bfloat16 else lib.ZO_F32
    r, dr = (r, dr) if residual else (None, None)
    y, h, dx, mean, rstd, dw, db = _outputs(x, w)
    ws = torch.empty(lib.zo_layernorm_workspace(rows, cols), dtype=torch.uint8, device=gpu)
    assert _forward(lib.LIB, lib, code, x, w, b, r, y, h, mean, rstd) == 0
    src = h if residual else x
    assert _backward(lib.LIB, lib, code, dy, src, w, mean, rstd, dr, dx, dw, db, ws) == 0
    lib.zo_layernorm_sync_status()
    for mode in range(6):
        assert probe.probe_lose(mode) == 0
        y1, h1, dx1, mean1, rstd1, dw1, db1 = _outputs(x, w)
        assert _forward(probe, lib, code, x, w, b, r, y1, h1, mean1, rstd1) == 0
        told = [probe.zo_layernorm_sync_status(None)]
        assert probe.zo_layernorm_sync_status(None) == lib.ZO_OK
        assert _backward(probe, lib, code, dy, src, w, mean, rstd, dr, dx1, dw1, db1, ws) == 0
        told.append(probe.zo_layernorm_sync_status(None))
        pairs = [(y1, y, True), (mean1, mean, True), (rstd1, rstd, True), (h1, h, False),
                 (dx1, dx, True), (dw1, dw, False), (db1, db, False)]
        for k, (got, right, by_rows) in enumerate(pairs):
            assert _right_or_nan(got, right, by_rows), (mode, k)
        # the status goes with the losses
        lost = [bool(torch.isnan(t).any()) for t in (y1, dx1)]
        assert told == [lib.ZO_ERR_TIMEOUT if n else lib.ZO_OK for n in lost], mode
        if rows * cols > 1 << 23 and dtype == torch.bfloat16 and not residual:
            assert lost == [mode != 0] * 2, mode         # rings in both passes, that go round
        # a row is NaN in all that is said of it
        assert torch.equal(torch.isnan(y1).any(1), torch.isnan(mean1))
    lib.zo_layernorm_sync_status()
