"""The norm's and the update's native calls against the binding's Python path on the same tensors: the same bits, shapes, strides and types; what is not
ordinary is left to the Python path, with its errors."""
import pytest
import torch

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    torch.cuda.set_device(0)


class _PythonPath:
    """Stands in for the native module and declines every call."""
    def __getattr__(self, name):
        return lambda *a: None


class _Counting:
    """The native module, counting the calls that it takes."""
    def __init__(self):
        self.module, self.taken = xb._load_native(), 0

    def __getattr__(self, name):
        def call(*a):
            out = getattr(self.module, name)(*a)
            self.taken += out is not None
            return out
        return call


FORMAT = {4: torch.channels_last, 5: torch.channels_last_3d}


def _make(shape, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype).contiguous(memory_format=FORMAT.get(len(shape), torch.contiguous_format))


def _flat(out):
    return [t for o in out for t in (o if isinstance(o, (list, tuple)) else [o])] if isinstance(out, (list, tuple)) else [out]


def _both(call, monkeypatch, taken):
    native = _Counting()
    monkeypatch.setattr(xb, "_native", native)
    got = _flat(call())
    assert native.taken == taken
    monkeypatch.setattr(xb, "_native", _PythonPath())
    want = _flat(call())
    assert len(got) == len(want)
    for a, b in zip(got, want):
        assert a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride() and torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(24,), (5, 40), (2, 3, 97), (2, 24, 5, 6), (1, 8, 3, 4, 5)])
def test_layer_norm(shape, dtype, monkeypatch):
    X, dY = _make(shape, dtype, 1), _make(shape, dtype, 2)
    C = shape[1] if len(shape) >= 4 else shape[-1]
    for w, b in ((_make((C,), dtype, 3), _make((C,), dtype, 4)), (_make((C,), torch.float32, 3), None), (None, None)):
        _both(lambda: xb.xconv_layernorm(X, w, b, 1e-3), monkeypatch, 1)
        _, mean, rstd = xb.xconv_layernorm(X, w, b)
        _both(lambda: xb.xconv_layernorm_backward(dY, X, mean, rstd, w), monkeypatch, 1)


def test_what_is_not_ordinary_goes_the_python_way(monkeypatch):
    X = _make((6, 40), torch.float32)
    w = _make((40,), torch.float32)
    _both(lambda: xb.xconv_layernorm(X[:, 1:30]), monkeypatch, 0)                # rows further apart than they are long
    _both(lambda: xb.xconv_layernorm(X, w, eps=1), monkeypatch, 0)               # an eps that is no float
    for call in (lambda: xb.xconv_layernorm(X, w[:39]), lambda: xb.xconv_layernorm(X, w.half()), lambda: xb.xconv_layernorm(X, w, w.cpu()),
                 lambda: xb.xconv_layernorm(X, _make((80,), torch.float32)[::2]), lambda: xb.xconv_layernorm(_make((2, 4, 3, 3), torch.float32).contiguous()),
                 lambda: xb.xconv_layernorm_backward(X, X, w, w), lambda: xb.xconv_layernorm_backward(X.half(), X, X[:, 0].contiguous(), X[:, 0].contiguous()),
                 lambda: xb.xconv_layernorm_backward(X, X, X[:, 0], X[:, 1].contiguous())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        xb.xconv_layernorm(X.double())
    with pytest.raises(xb.XConvError):
        xb.xconv_layernorm(X, w, eps=-1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_orthogonalize(dtype, monkeypatch):
    Gs = [_make(s, dtype, i) for i, s in enumerate([(20, 30), (2, 9, 8), (16, 8, 3, 3), (4, 4, 3, 3, 3)])]
    for G in Gs:
        _both(lambda: xb.xconv_orthogonalize(G), monkeypatch, 1)
    _both(lambda: xb.xconv_orthogonalize(Gs, steps=3, coefficients=(1.875, -1.25, 0.375), eps=1e-3), monkeypatch, 1)
    _both(lambda: xb.xconv_orthogonalize(tuple(Gs)), monkeypatch, 0)
    _both(lambda: xb.xconv_orthogonalize(Gs[0], coefficients=[1.875, -1.25, 0.375]), monkeypatch, 0)
    for bad in (Gs[0].T, Gs[0][0], Gs[2].contiguous(), Gs[0].cpu(), Gs + [Gs[0].T]):
        with pytest.raises(ValueError):
            xb.xconv_orthogonalize(bad)
    with pytest.raises(xb.XConvError):
        xb.xconv_orthogonalize(Gs[0], coefficients=(9.0, 0.0, 0.0))
    with pytest.raises(TypeError):
        xb.xconv_orthogonalize(Gs[0].double())


def test_muon_step(monkeypatch):
    shapes = [(20, 30), (2, 9, 8), (16, 8, 3, 3), (4, 4, 3, 3, 3)]
    wt = [torch.float32, torch.bfloat16, torch.float16, torch.float32]

    def step(single=False, **kw):
        W = [_make(s, t, i) for i, (s, t) in enumerate(zip(shapes, wt))]
        dW, M = [_make(s, torch.float32, i + 10) for i, s in enumerate(shapes)], [_make(s, torch.float32, i + 20) for i, s in enumerate(shapes)]
        if single:
            assert xb.xconv_muon_step(W[2], dW[2], M[2], 0.02, **kw) is W[2]
        else:
            assert xb.xconv_muon_step(W, dW, M, 0.02, **kw) is W
        return W, M

    _both(step, monkeypatch, 1)
    _both(lambda: step(single=True), monkeypatch, 1)
    _both(lambda: step(momentum=0.9, nesterov=False, weight_decay=0.1, steps=2, eps=1e-3, adjust="rms"), monkeypatch, 1)
    _both(lambda: step(momentum=0), monkeypatch, 0)
    W, dW, M = (_make((20, 30), torch.float32, i) for i in range(3))
    for args in ((W, dW, M.half()), (W, dW[:19], M), (W, [dW, dW], M), (W.T, dW.T, M.T)):
        with pytest.raises(ValueError):
            xb.xconv_muon_step(*args, 0.02)
    with pytest.raises(ValueError):
        xb.xconv_muon_step(W, dW, M, 0.02, adjust="no")
    for args in (([W, W], [dW, dW], [M, M]), (W, W, M), (W, dW, W)):             # a tensor that two of them write, or that one writes and another reads
        before = W.clone()
        with pytest.raises(xb.XConvError):
            xb.xconv_muon_step(*args, 0.02)
        assert torch.equal(W, before)


@pytest.mark.parametrize("native", [True, False])
def test_a_graph_that_keeps_the_weights_notices_the_step(native, monkeypatch):
    if not native:
        monkeypatch.setattr(xb, "_native", _PythonPath())
    W = _make((20, 30), torch.float32, 0).requires_grad_()
    x = _make((30, 4), torch.float32, 1).requires_grad_()
    y = (W @ x).sum()
    before = W._version
    M = torch.zeros_like(W.detach())
    xb.xconv_muon_step(W, torch.ones_like(W.detach()), M, 0.02)
    assert W._version > before and M._version > 0
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():                                    # (tensors without a count)
        W = torch.ones(20, 30, device="cuda")
        M = torch.zeros(20, 30, device="cuda")
        xb.xconv_muon_step(W, torch.ones(20, 30, device="cuda"), M, 0.02)
        assert W.isfinite().all() and not torch.equal(W, torch.ones_like(W))
