"""Layer norm at the limits of what one call may take for granted: other host threads, other calls on its scratch memory, the ends of the floats' range."""
import ctypes
import threading

import pytest
import torch

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("backward", [False, True])
def test_calls_of_different_sizes_from_two_host_threads(backward):
    """The same kernel with different amounts of shared memory (gradients: 48 and 96 KB; forward: 32 and 64 KB), by the C ABI's calls, which hold no lock of the interpreter's: no thread lowers
    the kernel's limit under another one's launch."""
    errors = []

    def job(rows):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                X = torch.randn(rows, 64, device="cuda").bfloat16()
                Y, mean, rstd = torch.empty_like(X), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
                dX, dw, db = torch.empty_like(X), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
                desc = xb.NormDesc(rows, 64, xb.XCONV_BF16, xb.XCONV_F32, 1e-5, 64, 64, 64)
                ws = torch.empty(xb.lib().xconv_layernorm_workspace_bytes(ctypes.byref(desc)), dtype=torch.uint8, device="cuda")
                p = [t.data_ptr() for t in (X, Y, mean, rstd, dX, dw, db, ws)]
                for i in range(4000):
                    if backward:
                        r = xb.lib().xconv_layernorm_backward(ctypes.byref(desc), p[0], p[0], p[2], p[3], None, p[4], p[5], p[6], p[7], ws.numel(), s.cuda_stream)
                    else:
                        r = xb.lib().xconv_layernorm_forward(ctypes.byref(desc), p[0], None, None, p[1], p[2], p[3], s.cuda_stream)
                    assert r == 0, (i, r, xb.lib().xconv_last_cuda_error())
                    if i % 100 == 0:
                        s.synchronize()
                s.synchronize()
        except BaseException as e:
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=job, args=(rows,)) for rows in (6000, 200000)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors, errors


def test_the_gradients_leave_the_scratch_memorys_header():
    """Two equal channels: their sums are the same bits, which in the header would read as a wait that ran out."""
    X = torch.randn(1000, 40, device="cuda")
    X[:, 1] = X[:, 0]
    dY = torch.randn(1000, 40, device="cuda")
    dY[:, 1] = dY[:, 0]
    _, mean, rstd = xb.xconv_layernorm(X)
    ws = xb.workspace(1 << 20, X.device)
    ws.zero_()
    assert xb.workspace_status(ws) == 0
    _, dw, db = xb.xconv_layernorm_backward(dY, X, mean, rstd)
    assert xb.workspace(1, X.device) is ws and dw[0] == dw[1] != 0 and db[0] == db[1] != 0
    assert xb.workspace_status(ws) == 0
    # what another call left there stays
    assert xb.lib().xconv_selftest_wait_limit(ws.data_ptr(), ws.numel(), 5, torch.cuda.current_stream().cuda_stream) == 0
    left = ws[:256].clone()
    xb.xconv_layernorm_backward(dY, X, mean, rstd)
    assert xb.workspace_status(ws) != 0 and torch.equal(ws[:256], left)


@pytest.mark.parametrize("eps,size", [(1e-5, 1.5e36), (1e-12, 1e33)])
@pytest.mark.parametrize("C", [7, 31, 97, 100, 601])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_large_rows_without_variance_are_finite(dtype, C, eps, size):
    """mean * rstd is beyond the floats there, (x - mean) * rstd is zero: also in the columns that a thread does not have."""
    rows = 70
    X = torch.full((rows, C), size, device="cuda").to(dtype)
    X[::2] *= -1
    mean, rstd = X[:, 0].float().contiguous(), torch.full((rows,), eps ** -0.5, device="cuda")
    assert not (mean * rstd).isfinite().any()
    dY = torch.randn(rows, C, device="cuda").to(dtype)
    dX, dw, db = xb.xconv_layernorm_backward(dY, X, mean, rstd)
    assert dX.isfinite().all() and (dw == 0).all()
    g = dY.double()
    want = rstd.double()[:, None] * (g - g.mean(1, keepdim=True))
    half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[dtype]
    # sums of up to 601 terms in chains of 150 at most, four operations behind them, one rounding to the type
    assert ((dX.double() - want).abs() <= half * want.abs() + (1 + half) * 154 * 2.0 ** -24 * rstd[:, None] * (g.abs() + g.abs().mean(1, keepdim=True))).all()
    assert ((db.double() - g.sum(0)).abs() <= rows * 2.0 ** -24 * g.abs().sum(0)).all()
