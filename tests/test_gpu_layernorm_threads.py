"""Layer norm called from several host threads at once, each on a stream and buffers of its own.
The calls share kernels whose dynamic shared memory differs with the width and the number of
matrices, and every one of them has to be launched whatever the others ask for."""

import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

# one instance's widths (512 threads a row), with more rows than are in flight at once
WIDTHS = (5200, 8000, 6100, 7300)
ROWS, CALLS = 330, 100


def _in_threads(work, n):
    failed, start = [], threading.Barrier(n)

    def run(k):
        try:
            start.wait()
            for _ in range(CALLS):
                status, why = work[k]()
                if status:
                    failed.append((k, status, why))
        except Exception as e:                              # noqa: BLE001 (reported below)
            failed.append((k, repr(e)))
    threads = [threading.Thread(target=run, args=(k,)) for k in range(n)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed[:8]


@pytest.mark.parametrize("passes", ["forward", "backward"])
def test_threads_with_other_widths(lib, gpu, passes):
    from paper_2608_15665_gb300 import firstorder as fo
    work, check, alive = [], [], []
    for k, n in enumerate(WIDTHS):
        g = torch.Generator().manual_seed(k)
        x, dy = (torch.randn(ROWS, n, generator=g).to(gpu) for _ in range(2))
        w = torch.ones(n, device=gpu)
        want = fo.layer_norm(x, w, None)
        grads = fo.layer_norm_backward(dy, x, w, want.mean, want.rstd)
        s = torch.cuda.Stream().cuda_stream
        out, mean, rstd = torch.zeros_like(x), torch.zeros_like(want.mean), torch.zeros_like(want.rstd)
        dw, db = torch.zeros_like(w), torch.zeros_like(w)
        ws = torch.empty(lib.zo_layernorm_workspace(ROWS, n), dtype=torch.uint8, device=gpu)
        alive.append((x, dy, w, want, grads, out, mean, rstd, dw, db, ws))
        if passes == "forward":
            args = (x.data_ptr(), n, None, 0, ROWS, n, lib.ZO_F32, w.data_ptr(), None, lib.ZO_F32,
                    1e-5, out.data_ptr(), n, None, 0, mean.data_ptr(), rstd.data_ptr(), s)
            work.append(lambda a=args: (lib.LIB.zo_layernorm_forward(*a), lib.zo_last_error()))
            check.append((want.y, out))
        else:
            args = (dy.data_ptr(), n, x.data_ptr(), n, None, 0, ROWS, n, lib.ZO_F32, w.data_ptr(),
                    lib.ZO_F32, want.mean.data_ptr(), want.rstd.data_ptr(), out.data_ptr(), n,
                    dw.data_ptr(), db.data_ptr(), ws.data_ptr(), ws.numel(), s)
            work.append(lambda a=args: (lib.LIB.zo_layernorm_backward(*a), lib.zo_last_error()))
            check += [(grads[0], out), (grads[1], dw), (grads[2], db)]
    torch.cuda.synchronize()
    _in_threads(work, len(WIDTHS))
    for want, got in check:
        assert torch.equal(want, got)
