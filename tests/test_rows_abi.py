"""Refusals of the entry points between the blocks and of their binding (no GPU: nothing is launched)."""
import ctypes
import os
import re

import pytest
import torch

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return xb.lib()


def _desc(**kw):
    base = dict(rows=6, C=40, dtype=xb.XCONV_BF16, param_dtype=xb.XCONV_F32, eps=1e-5, x_stride=40, r_stride=40, h_stride=40, dh_stride=40, y_stride=40, p=0.1, rows_per_mask=1)
    base.update(kw)
    return xb.RowsDesc(**base)


def _ref(d):
    return ctypes.byref(d) if d else None


def test_refusals_of_the_entry_points(lib):
    fwd = lambda d, X=16, R=16, w=16, H=16, Y=16, scales=None, rstd=16: lib.xconv_rmsnorm_forward(_ref(d), X, R, w, H, Y, scales, rstd, None)
    bwd = lambda d, dY=16, H=16, rstd=16, w=16, dH=16, dX=16, dR=16, dw=16, ws=16, n=1 << 40: lib.xconv_rmsnorm_backward(_ref(d), dY, H, rstd, w, dH, dX, dR, dw, ws, n, None)
    drop = lambda d, X=16, R=16, Y=16: lib.xconv_dropout(_ref(d), X, R, Y, None)
    deq = lambda d, Q=16, s=16, X=16: lib.xconv_dequantize(_ref(d), Q, s, X, None)
    q = dict(q_type=xb.XCONV_Q_E4M3)
    for call, more in ((fwd, {}), (bwd, {}), (drop, {}), (deq, q)):
        assert call(None) == 1
        for kw in (dict(rows=-3), dict(C=0), dict(C=-1), dict(dtype=3), dict(dtype=-1), dict(y_stride=-40), dict(x_stride=-1)):
            assert call(_desc(**{**more, **kw})) == 1, kw
        for kw in (dict(rows=1 << 40), dict(C=(1 << 30) + 8), dict(x_stride=1 << 61), dict(y_stride=1 << 61)):
            assert call(_desc(**{**more, **kw})) == 2, kw
    for call in (fwd, bwd):
        for kw in (dict(param_dtype=xb.XCONV_F16), dict(eps=-1e-5), dict(eps=float("nan")), dict(h_stride=-1)):
            assert call(_desc(**kw)) == 1, kw
        assert call(_desc(), w=18) == 3 and call(_desc(), rstd=18) == 3 and call(_desc(h_stride=1 << 61)) == 2
    for call in (fwd, bwd, drop):
        for kw in (dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(rows_per_mask=0), dict(rows_per_mask=-7)):
            assert call(_desc(**kw)) == 1, kw
        assert call(_desc(seed_add=20)) == 3
    assert fwd(_desc(), X=None) == 1 and fwd(_desc(), Y=None) == 1 and fwd(_desc(), X=17) == 3 and fwd(_desc(), R=17) == 3 and fwd(_desc(), H=17) == 3 and fwd(_desc(), Y=17) == 3
    assert fwd(_desc(y_stride=39)) == 1 and fwd(_desc(h_stride=39)) == 1
    assert fwd(_desc(), scales=16) == 1 and fwd(_desc(**q)) == 1 and fwd(_desc(q_type=3), scales=16) == 1 and fwd(_desc(**q, q_group=-1), scales=16) == 1
    assert fwd(_desc(**q, q_group=16), scales=16) == 2 and fwd(_desc(**q, q_group=39), scales=16) == 2 and fwd(_desc(**q), scales=18) == 3
    assert bwd(_desc(), dY=None) == 1 and bwd(_desc(), H=None) == 1 and bwd(_desc(), rstd=None) == 1 and bwd(_desc(), dX=None, dR=None, dw=None) == 1
    assert bwd(_desc(x_stride=39)) == 1 and bwd(_desc(r_stride=39)) == 1 and bwd(_desc(dh_stride=-1)) == 1
    for name in ("dY", "H", "dH", "dX", "dR", "dw"):
        assert bwd(_desc(), **{name: 17}) == 3, name
    need = lib.xconv_rmsnorm_workspace_bytes(ctypes.byref(_desc()))
    assert need >= 4 * 40
    assert bwd(_desc(), ws=None) == 4 and bwd(_desc(), n=need - 1) == 4 and bwd(_desc(), ws=24) == 3
    assert lib.xconv_rmsnorm_workspace_bytes(ctypes.byref(_desc(C=0))) == 0 and lib.xconv_rmsnorm_workspace_bytes(None) == 0
    assert drop(_desc(), X=None) == 1 and drop(_desc(), Y=None) == 1 and drop(_desc(y_stride=39)) == 1 and drop(_desc(), R=17) == 3
    assert deq(_desc()) == 1 and deq(_desc(**q), Q=None) == 1 and deq(_desc(**q), s=None) == 1 and deq(_desc(**q), X=None) == 1 and deq(_desc(**q), s=18) == 3
    assert deq(_desc(**q), X=17) == 3
    assert deq(_desc(**q, x_stride=39)) == 1 and deq(_desc(**q, q_group=8)) == 2


def test_no_rows_launch_nothing(lib):
    """(on a machine without a GPU a launch would fail)"""
    assert lib.xconv_rmsnorm_forward(_ref(_desc(rows=0)), 16, 16, 16, 16, 16, None, 16, None) == 0
    assert lib.xconv_dropout(_ref(_desc(rows=0)), 16, None, 16, None) == 0
    assert lib.xconv_dequantize(_ref(_desc(rows=0, q_type=2)), 16, 16, 16, None) == 0
    assert lib.xconv_rmsnorm_backward(_ref(_desc(rows=0)), 16, 16, 16, None, None, 16, None, None, None, 0, None) == 0
    assert lib.xconv_last_launch_count() == 0


def test_scratch_is_bounded_by_the_blocks_not_the_rows(lib):
    for C in (1, 24, 4096, 100000):
        sizes = [lib.xconv_rmsnorm_workspace_bytes(ctypes.byref(_desc(rows=r, C=C))) for r in (0, 1, 100, 10 ** 6, 2 * 10 ** 9)]
        assert sizes == sorted(sizes) and 0 < sizes[1] and sizes[-1] <= 256 + 148 * 16 * 4 * C


def test_the_binding_refuses_what_it_cannot_read(lib):
    t = torch.zeros(4, 8)
    q = torch.zeros(4, 8, dtype=torch.int8)
    for call in (lambda: xb.xconv_rmsnorm(t), lambda: xb.xconv_dropout(t, 0.1, 1), lambda: xb.xconv_dequantize(q, t), lambda: xb.xconv_rmsnorm_quantized(t),
                 lambda: xb.xconv_rmsnorm_backward(t, t, t[:, 0])):
        with pytest.raises(ValueError):
            call()                                         # host memory
    with pytest.raises(TypeError):
        xb.xconv_dequantize(t, t)
    with pytest.raises(TypeError):
        xb.xconv_rmsnorm_quantized(t, qdtype=torch.float8_e5m2)


class _Cuda(torch.Tensor):
    """A host tensor that says that it is on the GPU: it is looked at before anything is launched."""
    is_cuda = True


def test_the_bindings_arguments(lib, monkeypatch):
    monkeypatch.setattr(xb, "_elsewhere", lambda t: False)
    monkeypatch.setattr(xb, "_native", xb._Declines())
    c = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype).as_subclass(_Cuda)
    X = c(4, 64)
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(ValueError):
            xb.xconv_dropout(X, p, 1)
    with pytest.raises(ValueError):
        xb.xconv_dropout(X, 0.1, None)                     # no seed
    for residual in (c(4, 63), c(4, 64, dtype=torch.float16), c(2, 2, 64)):
        with pytest.raises(ValueError):
            xb.xconv_dropout(X, 0.1, 1, residual=residual)
        with pytest.raises(ValueError):
            xb.xconv_rmsnorm(X, residual=residual)
    for seed in (c(2, dtype=torch.int64), c(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int64)):
        with pytest.raises(ValueError):
            xb.xconv_dropout(X, 0.1, seed)
    for weight in (c(63), c(64, dtype=torch.float16), c(64, 1)):
        with pytest.raises(ValueError):
            xb.xconv_rmsnorm(X, weight)
    for group in (-1, 2 ** 31):
        with pytest.raises(ValueError):
            xb.xconv_rmsnorm_quantized(X, group=group)
    with pytest.raises(ValueError):
        xb.xconv_rmsnorm(c(4, 0))
    with pytest.raises(TypeError):
        xb.xconv_rmsnorm(c(4, 64, dtype=torch.float64))
    with pytest.raises(ValueError):
        xb.xconv_rmsnorm(torch.zeros(64, 4).t().as_subclass(_Cuda))
    Q = c(4, 64, dtype=torch.int8)
    for scales in (c(4), c(4, 2), c(4, 1, dtype=torch.float16), torch.zeros(4, 2)[:, :1].as_subclass(_Cuda)):
        with pytest.raises(ValueError):
            xb.xconv_dequantize(Q, scales)
    with pytest.raises(TypeError):
        xb.xconv_dequantize(Q, c(4, 1), dtype=torch.int32)
    for dY, rstd, dH in ((c(4, 63), c(4), None), (X, c(4, 1), None), (X, c(4, dtype=torch.float16), None), (X, c(4), c(3, 64))):
        with pytest.raises(ValueError):
            xb.xconv_rmsnorm_backward(dY, X, rstd, dH=dH)


def test_every_native_call_between_the_blocks_is_made_without_the_interpreters_lock():
    source = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2106_06998_b200", "csrc", "marshal.cpp")
    code = re.sub(r"//[^\n]*", "", open(source).read())
    names = re.findall(r"decltype\(&\w+\) (\w+);", code.split("struct RowsLibrary {")[1].split("}")[0])
    launching = [n for n in names if not n.endswith("workspace_bytes")]
    assert len(launching) == 4
    for n in launching:
        uses = [m.start() for m in re.finditer(r"\brows_lib\.%s\(" % n, code)]
        assert len(uses) == 1, n
        assert re.search(r"unlocked\(\[&\] \{\s*return $", code[:uses[0]]), n


def test_the_descriptor_is_as_the_header_has_it():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "xconv.h")).read()
    body = re.sub(r"/\*.*?\*/", "", header, flags=re.S).split("} xconv_rows_desc;")[0].split("typedef struct {")[-1]
    fields = [n.strip().lstrip("*") for line in re.findall(r"(?:int32_t|int64_t|float|double|unsigned long long|const unsigned long long\*) ([^;]+);", body) for n in line.split(",")]
    assert fields == [f[0] for f in xb.RowsDesc._fields_]
    assert ctypes.sizeof(xb.RowsDesc) == 8 + 6 * 4 + 5 * 8 + 8 + 8 + 8 + 8
