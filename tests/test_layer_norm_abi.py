"""Refusals of the layer norm's entry points and of its binding (no GPU: nothing is launched)."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return xb.lib()


def _desc(**kw):
    base = dict(rows=6, C=40, dtype=xb.XCONV_BF16, param_dtype=xb.XCONV_F32, eps=1e-5, x_stride=40, y_stride=40, dx_stride=40)
    base.update(kw)
    return xb.NormDesc(**base)


def test_refusals_of_the_entry_points(lib):
    fwd = lambda d, X=16, w=16, b=16, Y=16, mean=16, rstd=16: lib.xconv_layernorm_forward(ctypes.byref(d) if d else None, X, w, b, Y, mean, rstd, None)
    bwd = lambda d, dY=16, X=16, mean=16, rstd=16, w=16, dX=16, dw=16, db=16, ws=16, n=1 << 30: lib.xconv_layernorm_backward(
        ctypes.byref(d) if d else None, dY, X, mean, rstd, w, dX, dw, db, ws, n, None)
    for call in (fwd, bwd):
        assert call(None) == 1
        for kw in (dict(rows=0), dict(rows=-3), dict(C=0), dict(C=-1), dict(dtype=3), dict(dtype=-1), dict(param_dtype=xb.XCONV_F16), dict(eps=-1e-5),
                   dict(eps=float("nan")), dict(x_stride=-1), dict(y_stride=-40)):
            assert call(_desc(**kw)) == 1, kw
        for kw in (dict(rows=1 << 40), dict(C=(1 << 30) + 8), dict(x_stride=1 << 61)):
            assert call(_desc(**kw)) == 2, kw
        assert call(_desc(), X=None) == 1 and call(_desc(), X=17) == 3 and call(_desc(), w=18) == 3
    assert fwd(_desc(), Y=None) == 1 and fwd(_desc(), mean=None) == 1 and fwd(_desc(), rstd=None) == 1 and fwd(_desc(y_stride=39)) == 1
    assert fwd(_desc(), Y=15) == 3 and fwd(_desc(), mean=18) == 3 and fwd(_desc(), b=18) == 3
    assert bwd(_desc(), dY=None) == 1 and bwd(_desc(), mean=None) == 1 and bwd(_desc(), rstd=None) == 1 and bwd(_desc(), dX=None) == 1
    assert bwd(_desc(dx_stride=39)) == 1 and bwd(_desc(), dY=17) == 3 and bwd(_desc(), dw=18) == 3 and bwd(_desc(), ws=24) == 3
    need = lib.xconv_layernorm_workspace_bytes(ctypes.byref(_desc()))
    assert need >= 8 * 40
    assert bwd(_desc(), ws=None) == 4 and bwd(_desc(), n=need - 1) == 4
    assert lib.xconv_layernorm_workspace_bytes(ctypes.byref(_desc(C=0))) == 0


def test_scratch_is_bounded_by_the_blocks_not_the_rows(lib):
    for C in (1, 24, 4096, 100000):
        sizes = [lib.xconv_layernorm_workspace_bytes(ctypes.byref(_desc(rows=r, C=C, x_stride=C, y_stride=C, dx_stride=C))) for r in (1, 100, 10 ** 6, 2 * 10 ** 9)]
        assert sizes == sorted(sizes) and 0 < sizes[-1] <= 512 * 8 * C


def test_the_binding_refuses_what_it_cannot_read(lib):
    t = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        xb.xconv_layernorm(t)                              # host memory
    with pytest.raises(ValueError):
        xb.xconv_layernorm_backward(t, t, t[:, 0], t[:, 0])


class _Cuda(torch.Tensor):
    """A host tensor that says that it is on the GPU: its layout is looked at before anything is launched."""
    is_cuda = True


@pytest.mark.parametrize("shape,strides,want", [
    ((5, 8), (8, 1), ([5], 8, 8)), ((5, 8), (20, 1), ([5], 8, 20)), ((8,), (1,), ([], 8, 8)), ((1, 8), (100, 1), ([1], 8, 8)),
    ((2, 3, 8), (24, 8, 1), ([2, 3], 8, 8)), ((2, 3, 8), (60, 20, 1), ([2, 3], 8, 20)), ((2, 3, 8), (64, 20, 1), None), ((5, 8), (1, 5), None),
    ((2, 6, 4, 5), (120, 1, 30, 6), ([2, 4, 5], 6, 6)), ((2, 3, 4, 5), (120, 1, 30, 6), ([2, 4, 5], 3, 6)), ((2, 6, 4, 5), (120, 20, 5, 1), None),
    ((2, 3, 2, 4, 5), (240, 1, 120, 30, 6), ([2, 2, 4, 5], 3, 6)), ((2, 1, 4, 5), (20, 20, 5, 1), ([2, 4, 5], 1, 1)), ((1, 1, 1, 1, 1, 3), (3,) * 5 + (1,), None),
])
def test_rows_of_a_tensor(shape, strides, want):
    t = torch.empty_strided(shape, strides).as_subclass(_Cuda)
    if want is None:
        with pytest.raises(ValueError):
            xb._rows(t, "X")
    else:
        assert xb._rows(t, "X") == want
