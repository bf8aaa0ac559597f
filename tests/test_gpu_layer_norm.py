"""Layer norm, forward and backward, against its formulas in 64 bits: every type, rows on and off the 16-byte boundaries, from one value to more than a block's
registers hold, images, volumes, views of some channels, rows without variance and rows that are not finite."""
import threading

import pytest
import torch

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                      # half a step of a float
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    torch.cuda.set_device(0)


def last(t):
    """Channels last: (..., C)."""
    return t.movedim(1, -1) if t.dim() >= 4 else t


def make(shape, dtype, params, seed=0, offset=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    C = shape[1] if len(shape) >= 4 else shape[-1]
    fmt = {4: torch.channels_last, 5: torch.channels_last_3d}.get(len(shape), torch.contiguous_format)
    X = (rnd(*shape) + offset).to(dtype).contiguous(memory_format=fmt)
    dY = rnd(*shape).to(dtype).contiguous(memory_format=fmt)
    return X, dY, (1 + 0.3 * rnd(C)).to(params), (0.2 * rnd(C)).to(params)


def check_forward(X, w, b, Y, mean, rstd, eps=EPS):
    """A sum of n terms in chains of at most `depth` additions is off by at most depth * U times the sum of their sizes.  A thread adds up to 128 values of a
    register row (64 of a wide one here), ten steps of shuffles follow, four operations behind them."""
    depth = 150
    x = last(X).double()
    w = torch.ones(x.shape[-1], dtype=torch.float64, device="cuda") if w is None else w.double()
    b = torch.zeros_like(w) if b is None else b.double()
    m = x.mean(-1, keepdim=True)
    v = (x - m).square().mean(-1, keepdim=True)
    r = (v + eps).rsqrt()
    y = (x - m) * r * w + b
    dm = depth * U * x.abs().mean(-1, keepdim=True)
    assert ((mean.double().unsqueeze(-1) - m).abs() <= dm).all()
    rel = depth * U + (dm * r).square() + 2 * U * x.abs().amax(-1, keepdim=True) * r
    assert ((rstd.double().unsqueeze(-1) - r).abs() <= rel * r).all()
    tol = (dm + 2 * U * x.abs()) * r * w.abs() + rel * ((x - m) * r * w).abs() + 4 * U * (b.abs() + y.abs())
    tol = tol * 1.01 + HALF[X.dtype] * (y.abs() + tol) + (2.0 ** -25 if X.dtype == torch.float16 else 0)      # (half a step of a subnormal float16)
    assert ((last(Y).double() - y).abs() <= tol).all(), float(((last(Y).double() - y).abs() / tol).max())


def check_backward(dY, X, mean, rstd, w, dX, dw, db):
    """mean and rstd are inputs.  xh is off by 3 U of itself and U |x| rstd (the difference); each of the two sums over a row by depth * U of its terms' sizes."""
    depth = 150
    x, dy = last(X).double(), last(dY).double()
    C = x.shape[-1]
    m, r = mean.double().unsqueeze(-1), rstd.double().unsqueeze(-1)
    w = torch.ones(C, dtype=torch.float64, device="cuda") if w is None else w.double()
    xh = (x - m) * r
    dxh = 3 * U * xh.abs() + U * (x - m).abs() * r
    g = dy * w
    m0, m1 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    want = r * (g - m0 - xh * m1)
    e0 = depth * U * g.abs().mean(-1, keepdim=True)
    e1 = depth * U * (g * xh).abs().mean(-1, keepdim=True) + (g.abs() * dxh).mean(-1, keepdim=True)
    tol = r * (4 * U * g.abs() + e0 + 4 * U * m0.abs() + xh.abs() * e1 + dxh * m1.abs() + 4 * U * (xh * m1).abs())
    tol = 1.01 * tol + HALF[X.dtype] * (want.abs() + tol) + (2.0 ** -25 if X.dtype == torch.float16 else 0)
    err = (last(dX).double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())
    # a thread adds up to rows / 148 products, 16 teams of a block follow, then up to 512 parts in 32 lanes
    flat = lambda t: t.reshape(-1, C).sum(0)
    n = x.numel() // C
    chain = n / 100 + 16 + 16 + 20
    assert ((dw.double() - flat(dy * xh)).abs() <= (chain + 4) * U * flat((dy * xh).abs()) + flat(dy.abs() * dxh)).all()
    assert ((db.double() - flat(dy)).abs() <= (chain + 4) * U * flat(dy.abs())).all()


SHAPES = [(1, 1), (1, 2), (3, 1), (1, 4096), (5, 7), (33, 97), (9, 24), (257, 1000), (64, 2257), (7, 8192), (5, 4100), (3, 8200), (2, 16392), (4, 9001), (2, 40001),
          (6, 520), (70001, 8), (4099, 96), (2, 3, 5, 7), (3, 64, 9, 5), (2, 130, 6, 6), (1, 24, 3, 5, 7), (2, 17, 4, 3, 2), (4, 9, 40), (12,), (300, 1536),
          # dense rows that do not begin on 16-byte boundaries, enough for runs, a last run that is not whole; odd and even numbers of values
          (4099, 97), (999, 33), (5003, 7), (3001, 201), (777, 1), (1235, 98), (2001, 2), (601, 2047), (50, 97, 9, 7)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", SHAPES)
def test_layer_norm_of_any_shape(shape, dtype):
    for params in {torch.float32, dtype}:
        X, dY, w, b = make(shape, dtype, params, seed=len(shape) + shape[-1])
        Y, mean, rstd = xb.xconv_layernorm(X, w, b, eps=EPS)
        assert Y.shape == X.shape and Y.dtype == dtype and mean.dtype == rstd.dtype == torch.float32 and list(mean.shape) == list(last(X).shape[:-1])
        check_forward(X, w, b, Y, mean, rstd)
        dX, dw, db = xb.xconv_layernorm_backward(dY, X, mean, rstd, w)
        assert dX.shape == X.shape and dX.dtype == dtype and dw.dtype == db.dtype == torch.float32 and dw.shape == db.shape == w.shape
        check_backward(dY, X, mean, rstd, w, dX, dw, db)


@pytest.mark.parametrize("shape", [(33, 97), (65, 512), (3, 64, 9, 5)])
def test_without_parameters(shape):
    X, dY, w, b = make(shape, torch.bfloat16, torch.float32)
    for weight, bias in ((None, None), (w, None), (None, b)):
        Y, mean, rstd = xb.xconv_layernorm(X, weight, bias, eps=EPS)
        check_forward(X, weight, bias, Y, mean, rstd)
    out = xb.xconv_layernorm_backward(dY, X, mean, rstd)
    check_backward(dY, X, mean, rstd, None, *out)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("first,count", [(0, 64), (8, 40), (1, 33), (3, 1)])
def test_views_of_some_channels(dtype, first, count):
    """Rows that lie further apart than they are long, on and off the 16-byte boundaries; nothing beside them enters or is written."""
    for shape in ((45, 80), (3, 7, 80), (2, 80, 6, 5)):
        X, dY, w, b = make(shape, dtype, torch.float32)
        cut = (lambda t: t[:, first:first + count]) if len(shape) == 4 else (lambda t: t[..., first:first + count])
        out = xb.xconv_layernorm(cut(X), w[:count].contiguous(), b[:count].contiguous(), eps=EPS)
        check_forward(cut(X), w[:count], b[:count], *out)
        grads = xb.xconv_layernorm_backward(cut(dY), cut(X), out[1], out[2], w[:count].contiguous())
        check_backward(cut(dY), cut(X), out[1], out[2], w[:count], *grads)


def test_rows_further_apart_than_32_bits_reach():
    """The last of 70 000 rows begins 2.8 thousand million elements behind the first."""
    wide = torch.empty((70000, 40000), dtype=torch.bfloat16, device="cuda")
    X, dY, w, b = make((70000, 64), torch.bfloat16, torch.float32)
    view = wide[:, 24:88]
    view.copy_(X)
    Y, mean, rstd = xb.xconv_layernorm(view, w, b, eps=EPS)
    Yd, md, rd = xb.xconv_layernorm(X, w, b, eps=EPS)
    assert torch.equal(Y, Yd) and torch.equal(mean, md) and torch.equal(rstd, rd)
    for got, want in zip(xb.xconv_layernorm_backward(dY, view, mean, rstd, w), xb.xconv_layernorm_backward(dY, X, md, rd, w)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("C", [8, 97, 1024, 9000])
def test_rows_without_variance(C):
    """Every value the same: the difference to the mean is a rounding of the mean at most, over sqrt(eps) -- for values that are sums of few powers of two it is 0."""
    X = torch.full((5, C), 3.0, device="cuda")
    Y, mean, rstd = xb.xconv_layernorm(X, eps=EPS)
    check_forward(X, None, None, Y, mean, rstd)
    Y, mean, rstd = xb.xconv_layernorm(torch.zeros_like(X), eps=EPS)
    assert (Y == 0).all() and (mean == 0).all() and torch.allclose(rstd, torch.full_like(rstd, EPS ** -0.5), rtol=1e-6)
    dX, dw, db = xb.xconv_layernorm_backward(torch.ones_like(X), torch.zeros_like(X), mean, rstd)
    assert (dw == 0).all() and (db == 5).all()


def test_a_large_mean_does_not_cost_the_variance():
    """Differences to the mean, not a difference of sums of squares: 1000 times the standard deviation above zero, rstd keeps three digits less than a float has."""
    X, _, _, _ = make((40, 768), torch.float32, torch.float32, offset=1000.0)
    check_forward(X, None, None, *xb.xconv_layernorm(X, eps=EPS))


@pytest.mark.parametrize("C", [64, 97, 4096, 9000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_row_that_is_not_finite_is_the_only_one(C, bad):
    X, dY, w, b = make((21, C), torch.float16, torch.float32)
    fine = xb.xconv_layernorm(X, w, b, eps=EPS)
    gfine = xb.xconv_layernorm_backward(dY, X, *fine[1:], w)
    X[7, C // 2] = bad
    Y, mean, rstd = xb.xconv_layernorm(X, w, b, eps=EPS)
    others = [i for i in range(21) if i != 7]
    assert Y[7].isnan().all() and not mean[7].isfinite() and rstd[7].isnan()
    assert torch.equal(Y[others], fine[0][others]) and torch.equal(mean[others], fine[1][others]) and torch.equal(rstd[others], fine[2][others])
    dX, dw, db = xb.xconv_layernorm_backward(dY, X, mean, rstd, w)
    assert dX[7].isnan().all() and torch.equal(dX[others], gfine[0][others]) and dw.isnan().all() and torch.equal(db, gfine[2])


def test_gradients_against_differences():
    """Central differences of the library's own forward pass: their error is h^2 / 6 times a third derivative (below 60 here) and the roundings of the loss over h."""
    X, dY, w, b = make((3, 24), torch.float32, torch.float32, seed=5)
    _, mean, rstd = xb.xconv_layernorm(X, w, b, eps=EPS)
    dX, dw, db = xb.xconv_layernorm_backward(dY, X, mean, rstd, w)
    h = 2.0 ** -6
    loss = lambda x, ww, bb: float((xb.xconv_layernorm(x, ww, bb, eps=EPS)[0].double() * dY.double()).sum())
    tol = 60 * h * h / 6 + 3 * 24 * 16 * U / h
    for t, grad in ((X, dX), (w, dw), (b, db)):
        for i in range(0, t.numel(), 5):
            up, down = t.clone(), t.clone()
            up.view(-1)[i] += h
            down.view(-1)[i] -= h
            args = [(up if u is t else u, down if u is t else u) for u in (X, w, b)]
            diff = (loss(*[p[0] for p in args]) - loss(*[p[1] for p in args])) / (2 * h)
            assert abs(diff - float(grad.view(-1)[i])) <= tol


def test_the_same_bits_again_on_other_streams_and_from_a_graph():
    X, dY, w, b = make((8, 96, 14, 14), torch.bfloat16, torch.float32)

    def step():
        Y, mean, rstd = xb.xconv_layernorm(X, w, b, eps=EPS)
        return (Y, mean, rstd) + xb.xconv_layernorm_backward(dY, X, mean, rstd, w)

    want = step()
    torch.cuda.synchronize()
    got, errors = [], []

    def job():
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(20):
                    out = step()
            s.synchronize()
            got.append(out)
        except Exception as e:
            errors.append(e)

    threads = [threading.Thread(target=job) for _ in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors and len(got) == 4
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for t in captured:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for out in got + [captured]:
        assert all(torch.equal(g, t) for g, t in zip(out, want))


def test_rows_behind_the_last_are_left_as_they_were():
    """Outputs that are the front of a larger buffer."""
    import ctypes
    for C, dtype in ((97, torch.float16), (64, torch.bfloat16), (9001, torch.float32)):
        X, dY, w, b = make((19, C), dtype, torch.float32)
        out = torch.full((40, C), 7.0, dtype=dtype, device="cuda")
        stats = torch.full((2, 40), 7.0, device="cuda")
        sums = torch.full((2, 2 * C), 7.0, device="cuda")
        d = xb.NormDesc(19, C, xb._dtype_code(dtype), xb.XCONV_F32, EPS, C, C, C)
        L = xb.lib()
        ws = torch.empty(L.xconv_layernorm_workspace_bytes(ctypes.byref(d)), dtype=torch.uint8, device="cuda")
        s = xb._stream()
        assert L.xconv_layernorm_forward(ctypes.byref(d), X.data_ptr(), w.data_ptr(), b.data_ptr(), out.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(), s) == 0
        check_forward(X, w, b, out[:19], stats[0, :19], stats[1, :19])
        assert (out[19:] == 7).all() and (stats[:, 19:] == 7).all()
        out.fill_(7.0)
        assert L.xconv_layernorm_backward(ctypes.byref(d), dY.data_ptr(), X.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(), w.data_ptr(), out.data_ptr(),
                                          sums[0].data_ptr(), sums[1].data_ptr(), ws.data_ptr(), ws.numel(), s) == 0
        check_backward(dY, X, stats[0, :19], stats[1, :19], w, out[:19], sums[0, :C], sums[1, :C])
        assert (out[19:] == 7).all() and (sums[:, C:] == 7).all()
        # what is not asked for is not written
        sums.fill_(7.0)
        assert L.xconv_layernorm_backward(ctypes.byref(d), dY.data_ptr(), X.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(), w.data_ptr(), out.data_ptr(),
                                          None, sums[1].data_ptr(), ws.data_ptr(), ws.numel(), s) == 0
        assert (sums[0] == 7).all() and (sums[1, :C] != 7).any()
        assert L.xconv_layernorm_backward(ctypes.byref(d), dY.data_ptr(), X.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(), w.data_ptr(), out.data_ptr(),
                                          None, None, None, 0, s) == 0
        check_backward(dY, X, stats[0, :19], stats[1, :19], w, out[:19], *xb.xconv_layernorm_backward(dY, X, stats[0, :19], stats[1, :19], w)[1:])


@pytest.mark.parametrize("C", [97, 136])
def test_offsets_that_pass_32_bits(C):
    """Rows of zeros (whose gradients are zeros, and add nothing to the columns' sums) before the ones that are looked at."""
    tail = 2000
    rows = 2 ** 32 // C + tail + 5
    X, dY = (torch.zeros((rows, C), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x, dy, w, b = make((tail, C), torch.bfloat16, torch.float32, seed=C)
    X[-tail:], dY[-tail:] = x, dy
    Y, mean, rstd = xb.xconv_layernorm(X, w, b, eps=EPS)
    check_forward(x, w, b, Y[-tail:], mean[-tail:], rstd[-tail:])
    assert torch.equal(Y[:-tail].amin(0), b.bfloat16()) and torch.equal(Y[:-tail].amax(0), b.bfloat16()) and not mean[:-tail].any()
    del Y
    dX, dw, db = xb.xconv_layernorm_backward(dY, X, mean, rstd, w)
    check_backward(dy, x, mean[-tail:], rstd[-tail:], w, dX[-tail:], dw, db)
    assert not dX[:-tail].amax(0).any() and not dX[:-tail].amin(0).any()


@pytest.mark.parametrize("at, C", [(4096, 1000), (4097, 97), (64, 20000)])
def test_strides_whose_offsets_pass_32_bits(at, C):
    buffer = torch.empty((35, 2 ** 27), dtype=torch.bfloat16, device="cuda")
    x, dy, w, b = make((35, C), torch.bfloat16, torch.bfloat16, seed=at)
    X, dY = buffer[:, at:at + C], buffer[:, 2 ** 26 + at:2 ** 26 + at + C]
    X.copy_(x); dY.copy_(dy)
    Y, mean, rstd = xb.xconv_layernorm(X, w, b, eps=EPS)
    check_forward(x, w, b, Y, mean, rstd)
    check_backward(dy, x, mean, rstd, w, *xb.xconv_layernorm_backward(dY, X, mean, rstd, w))
