"""Dropout from a seed, RMS norm with a residual, its gradients and its 8-bit outputs against their formulas in 64 bits."""
import ctypes

import pytest
import torch

from paper_2106_06998_b200 import binding as xb
from tests import _rows as R

pytestmark = pytest.mark.gpu

T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SEED = 0x1234_5678_9ABC_DEF1


def tensor(shape, dtype, seed, kind="dense", scale=1.0):
    """A tensor of the library's layout: dense, some channels of a wider one that begin on an odd one ("cut") or on a 16-byte boundary ("wide"), or off 16 bytes ("shifted")."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    C = shape[1] if len(shape) >= 4 else shape[-1]
    rows = [s for i, s in enumerate(shape) if i != (1 if len(shape) >= 4 else len(shape) - 1)]
    extra, first = {"dense": (0, 0), "cut": (5, 3), "wide": (16, 8), "shifted": (0, 0)}[kind]
    n = 1
    for s in rows:
        n *= s
    flat = (torch.randn(n * (C + extra) + 1, generator=gen, device="cuda") * scale).to(dtype)
    base = flat[1:] if kind == "shifted" else flat[:-1]
    t = base.view(*rows, C + extra)[..., first:first + C]
    return t.movedim(-1, 1) if len(shape) >= 4 else t


SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 8), (1000, 12), (33, 129), (7, 300), (19, 1000), (40, 2056), (9, 8192), (3, 8200), (2, 16385), (2, 40001), (700,), (4, 6, 72),
          (2, 16, 5, 7), (3, 97, 9, 11), (2, 20, 3, 4, 5), (300, 64), (257, 31)]
KINDS = ["dense", "cut", "wide", "shifted"]


def cases():
    out = []
    for i, shape in enumerate(SHAPES):
        for j, t in enumerate(T):
            out.append((shape, t, KINDS[(i + j) % 4] if len(shape) > 1 else "dense", (i + j) % 2 == 0))
    return out


@pytest.mark.parametrize("shape,dtype,kind,own_params", cases())
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_rmsnorm(shape, dtype, kind, own_params, p):
    t = T[dtype]
    C = shape[1] if len(shape) >= 4 else shape[-1]
    X, residual = tensor(shape, t, 1, kind), tensor(shape, t, 2, "dense" if kind == "cut" else kind, 3.0)
    weight = tensor((C,), t if own_params else torch.float32, 3)
    for r, w in ((residual, weight), (None, None)):
        Y, H, rstd = xb.xconv_rmsnorm(X, w, residual=r, eps=1e-5, p=p, seed=SEED)
        (y, h, s), (y_off, h_off, s_off) = R.norm(X, w, r, 1e-5, p, SEED)
        R.close("Y", R.last(Y), y, R.rounded(y, y_off, t))
        R.close("rstd", rstd.cpu().double().reshape(-1), s, s_off + 2.0 ** -23 * s)
        assert Y.shape == X.shape and Y.dtype == t and (H is X if r is None and p == 0 else True)
        R.close("H", R.last(H), h, R.rounded(h, h_off, t))


@pytest.mark.parametrize("shape,dtype,kind,own_params", cases())
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_rmsnorm_backward(shape, dtype, kind, own_params, p):
    t = T[dtype]
    C = shape[1] if len(shape) >= 4 else shape[-1]
    H, dY, dH = tensor(shape, t, 1, "dense" if kind == "cut" else kind, 2.0), tensor(shape, t, 2, kind), tensor(shape, t, 4, kind)
    weight = tensor((C,), t if own_params else torch.float32, 3)
    rstd = (H.float().movedim(1, -1) if H.dim() >= 4 else H.float()).square().mean(-1).add(1e-5).rsqrt().contiguous()
    for d, w in ((dH, weight), (None, None)):
        dX, dR, dw = xb.xconv_rmsnorm_backward(dY, H, rstd, w, dH=d, p=p, seed=SEED)
        (dx, dr, dweight), (x_off, r_off, w_off) = R.norm_backward(dY, H, rstd, w, d, p, SEED)
        R.close("dresidual", R.last(dR), dr, R.rounded(dr, r_off, t))
        R.close("dX", R.last(dX), dx, R.rounded(dx, x_off, t))
        R.close("dweight", dw.cpu().double(), dweight, w_off + 2.0 ** -24 * dweight.abs())
        assert (dR is dX) == (p == 0)
        again = xb.xconv_rmsnorm_backward(dY, H, rstd, w, dH=d, p=p, seed=SEED)
        assert all(torch.equal(a, b) for a, b in zip((dX, dR, dw), again))


@pytest.mark.parametrize("rows,C", [(20000, 40), (3000, 1024), (9000, 97)])
def test_many_rows(rows, C):
    H, dY = tensor((rows, C), torch.bfloat16, 1), tensor((rows, C), torch.bfloat16, 2)
    Y, _, rstd = xb.xconv_rmsnorm(H)
    (y, _, _), (y_off, _, _) = R.norm(H, None, None, 1e-6)
    R.close("Y", R.last(Y), y, R.rounded(y, y_off, torch.bfloat16))
    dX, _, dw = xb.xconv_rmsnorm_backward(dY, H, rstd)
    (dx, _, dweight), (x_off, _, w_off) = R.norm_backward(dY, H, rstd, None, None)
    R.close("dX", R.last(dX), dx, R.rounded(dx, x_off, torch.bfloat16))
    R.close("dweight", dw.cpu().double(), dweight, w_off)


@pytest.mark.parametrize("shape,dtype,kind,_", cases())
@pytest.mark.parametrize("channels", [False, True])
def test_dropout(shape, dtype, kind, _, channels):
    t = T[dtype]
    X, residual = tensor(shape, t, 1, kind), tensor(shape, t, 2, kind, 3.0)
    for p in (0.1, 0.5, 1.0, 0.0):
        Y = xb.xconv_dropout(X, p, SEED, channels=channels)
        want = R.dropped(R.last(X), p, SEED, R.per_of(X, channels))
        R.close("Y", R.last(Y), want, R.rounded(want, 2.0 ** -23 * want.abs(), t))
        assert torch.equal(Y, xb.xconv_dropout_backward(X, p, SEED, channels=channels))
        Y = xb.xconv_dropout(X, p, SEED, residual=residual, channels=channels)
        off = 2.0 ** -22 * (want.abs() + R.last(residual).abs())
        want = want + R.last(residual)
        R.close("Y", R.last(Y), want, R.rounded(want, off, t))


@pytest.mark.parametrize("p", [1e-4, 0.25, 0.1, 1 - 2.0 ** -20, 2.0 ** -32, 3 * 2.0 ** -17])
def test_the_mask_to_the_last_bit(p):
    """Four million values: some 64 of them have the upper half of the border, and the lower half decides."""
    X = torch.ones(4096, 1024, device="cuda")
    for seed in (0, 2 ** 64 - 1, -5):
        got = xb.xconv_dropout(X, p, seed) != 0
        assert torch.equal(got.cpu(), R.kept(4096, 1024, p, seed))


def test_a_dropped_value_is_zero_whatever_it_was():
    X = torch.full((64, 64), float("nan"), device="cuda")
    X[::2] = float("inf")
    Y = xb.xconv_dropout(X, 0.5, 7).cpu()
    mask = R.kept(64, 64, 0.5, 7)
    assert bool((Y[~mask] == 0).all()) and bool(torch.isnan(Y[1::2][mask[1::2]]).all()) and bool(torch.isinf(Y[::2][mask[::2]]).all())
    assert bool((xb.xconv_dropout(X, 1.0, 7) == 0).all())


def test_values_that_pass_32_bits():
    """The mask of rows far down in a tensor of more than 2^31 values."""
    X = torch.ones(2 ** 27 + 5, 17, dtype=torch.bfloat16, device="cuda")
    Y = xb.xconv_dropout(X, 0.5, 3)
    first = 2 ** 27 - 20
    assert torch.equal((Y[first:] != 0).cpu(), R.kept(25, 17, 0.5, 3, first=first))


@pytest.mark.parametrize("C", [16, 17])
def test_norms_of_values_that_pass_32_bits(C):
    """The last rows of more than 2^31 values, and the columns' sums over all of them (of ones: their number, which floats hold)."""
    rows, t = 2 ** 27 + 6, torch.bfloat16
    X = torch.ones(rows, C, dtype=t, device="cuda")
    tail = tensor((20, C), t, 1)
    X[-20:] = tail
    Y, H, rstd = xb.xconv_rmsnorm(X, p=0.25, seed=3)
    mask = R.kept(20, C, 0.25, 3, first=rows - 20)
    x = torch.where(mask, R.last(tail) / 0.75, torch.zeros((), dtype=torch.float64))
    (y, h, s), (y_off, h_off, s_off) = R.norm(x, None, None, 1e-6)
    R.close("H", R.last(H[-20:]), h, R.rounded(h, h_off, t))
    R.close("Y", R.last(Y[-20:]), y, R.rounded(y, y_off + h_off * s[:, None], t))
    del Y, H
    Q, scales, _, _ = xb.xconv_rmsnorm_quantized(X, qdtype=torch.int8)
    (y, _, _), (y_off, _, _) = R.norm(tail, None, None, 1e-6)
    codes, wide = check_8_bits(Q[-20:], scales[-20:], y, y_off, C, 127.0)
    V = xb.xconv_dequantize(Q, scales, dtype=t)
    R.close("V", R.last(V[-20:]), codes * wide, R.rounded(codes * wide, 0 * wide, t))
    del Q, V
    ones = torch.ones(rows, device="cuda")
    dX, _, dw = xb.xconv_rmsnorm_backward(X, X, ones)
    (dx, _, _), (x_off, _, _) = R.norm_backward(X[-20:], X[-20:], ones[-20:], None, None)
    R.close("dX", R.last(dX[-20:]), dx, R.rounded(dx, x_off, t))
    want = rows - 20 + R.last(tail).square().sum(0)
    # (threads add some 2^27 / 2^15 numbers one after another, each with a rounding of 2^-24 of what is there by then)
    R.close("dweight", dw.cpu().double(), want, 2.0 ** -11 * want)


def _seed_tensor(v):
    return torch.tensor([v], dtype=torch.int64, device="cuda")


def test_a_seed_in_device_memory():
    X = tensor((50, 200), torch.bfloat16, 1)
    for v in (0, 12345, -3, 2 ** 62):
        assert torch.equal(xb.xconv_dropout(X, 0.3, _seed_tensor(v)), xb.xconv_dropout(X, 0.3, v))
    Y, H, rstd = xb.xconv_rmsnorm(X, p=0.3, seed=_seed_tensor(5))
    assert torch.equal(H, xb.xconv_dropout(X, 0.3, 5))
    dX, dR, dw = xb.xconv_rmsnorm_backward(X, H, rstd, p=0.3, seed=_seed_tensor(5))
    assert torch.equal(xb.xconv_rmsnorm_backward(X, H, rstd, p=0.3, seed=5)[0], dX)


def test_a_captured_step_draws_another_mask_in_every_replay():
    X, res, w = tensor((64, 320), torch.float32, 1), tensor((64, 320), torch.float32, 2), tensor((320,), torch.float32, 3)
    seed = _seed_tensor(100)

    def step():
        Y, H, rstd = xb.xconv_rmsnorm(X, w, residual=res, p=0.2, seed=seed)
        out = (Y, H, *xb.xconv_rmsnorm_backward(Y, H, rstd, w, dH=H, p=0.2, seed=seed))
        seed.add_(1)
        return out

    step()
    torch.cuda.synchronize()
    seed.fill_(100)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    seed.fill_(100)
    before = None
    for _ in range(3):
        value = int(seed)
        graph.replay()
        torch.cuda.synchronize()
        saved = [t.clone() for t in got]
        seed.fill_(value)
        for a, b in zip(saved, step()):
            assert torch.equal(a, b)
        assert before is None or not torch.equal(before, saved[1])
        before = saved[1]


def e4m3_half_step(v):
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    return torch.exp2(e - 4)


def check_8_bits(Q, scales, y, y_off, width, M):
    """Codes and scales of y, of `width` values a scale; returns both in 64 bits."""
    C = y.shape[1]
    pad = lambda v: torch.nn.functional.pad(v, (0, -C % width)).reshape(v.shape[0], -1, width)
    most, most_off = pad(y).abs().amax(-1), pad(y_off).amax(-1)
    got = R.last(scales)
    R.close("scales", got, most.clamp(min=2.0 ** -100) / M, (most_off + 2.0 ** -22 * most) / M + 2.0 ** -140)
    wide, codes = got.repeat_interleave(width, 1)[:, :C], R.last(Q.float())
    assert float(codes.abs().max()) <= M
    # the nearest 8-bit value: half a step, where the value before it may be off by what float arithmetic is, and by the product with 1 / scale
    half = e4m3_half_step(codes) if M == 448.0 else torch.full_like(codes, 0.5)
    R.close("Q", codes, y / wide, half + y_off / wide + 2.0 ** -21 * (y / wide).abs())
    return codes, wide


@pytest.mark.parametrize("shape,dtype,kind,own_params", cases())
@pytest.mark.parametrize("q", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
def test_rmsnorm_in_8_bits(shape, dtype, kind, own_params, q, group):
    t = T[dtype]
    C = shape[1] if len(shape) >= 4 else shape[-1]
    X, residual = tensor(shape, t, 1, kind), tensor(shape, t, 2, "dense" if kind == "cut" else kind, 3.0)
    weight = tensor((C,), t if own_params else torch.float32, 3)
    Q, scales, H, rstd = xb.xconv_rmsnorm_quantized(X, weight, residual=residual, eps=1e-5, qdtype=q, group=group)
    (y, h, s), (y_off, h_off, s_off) = R.norm(X, weight, residual, 1e-5)
    R.close("H", R.last(H), h, R.rounded(h, h_off, t))
    R.close("rstd", rstd.cpu().double().reshape(-1), s, s_off + 2.0 ** -23 * s)
    width = group if 0 < group < C else C
    codes, wide = check_8_bits(Q, scales, y, y_off, width, 448.0 if q == torch.float8_e4m3fn else 127.0)
    assert Q.dtype == q and Q.shape == X.shape
    for out in (torch.float32, torch.bfloat16, torch.float16):
        V = xb.xconv_dequantize(Q, scales, group=group, dtype=out)
        want = codes * wide
        assert V.dtype == out and V.shape == X.shape
        R.close("V", R.last(V), want, R.rounded(want, 0 * want, out))


def test_8_bits_of_rows_that_are_zero_small_or_not_finite():
    X = tensor((6, 256), torch.float32, 1)
    X[0] = 0; X[1] *= 1e-30; X[3, 7] = float("nan"); X[4, 200] = float("inf")
    w = torch.ones(256, device="cuda"); w[40] = 1e-38
    for q in (torch.float8_e4m3fn, torch.int8):
        for group in (0, 32):
            Q, scales, _, rstd = xb.xconv_rmsnorm_quantized(X, w, eps=1e-6, qdtype=q, group=group)
            V = xb.xconv_dequantize(Q, scales, group=group, dtype=torch.float32)
            assert bool((V[0] == 0).all()) and bool((scales[0] > 0).all())
            assert bool(torch.isnan(V[3]).all())                 # (its rstd is NaN)
            at = slice(192, 224) if group else slice(0, 256)
            assert bool(torch.isnan(V[4, at]).all())             # (rstd = 0: infinity times zero)
            assert bool(torch.isfinite(V[[0, 1, 2, 5]]).all())
            clean, _, _, _ = xb.xconv_rmsnorm_quantized(X[[5]], w, eps=1e-6, qdtype=q, group=group)
            assert torch.equal(Q[5].view(torch.uint8), clean[0].view(torch.uint8))


def test_not_finite_values_stay_in_their_rows():
    X, dY = tensor((40, 72), torch.bfloat16, 1), tensor((40, 72), torch.bfloat16, 2)
    Y0, _, r0 = xb.xconv_rmsnorm(X)
    dX0, _, _ = xb.xconv_rmsnorm_backward(dY, X, r0)
    X[7, 3] = float("nan"); X[21, 70] = float("-inf")
    Y, _, r = xb.xconv_rmsnorm(X)
    dX, _, dw = xb.xconv_rmsnorm_backward(dY, X, r)
    others = [i for i in range(40) if i not in (7, 21)]
    assert torch.equal(Y[others], Y0[others]) and torch.equal(dX[others], dX0[others])
    assert bool(torch.isnan(Y[7]).all()) and bool(torch.isnan(Y[21, 70])) and bool(torch.isnan(dw).all())


def test_no_rows():
    X, w = torch.empty(0, 40, device="cuda", dtype=torch.bfloat16), torch.ones(40, device="cuda")
    Y, H, rstd = xb.xconv_rmsnorm(X, w, residual=X, p=0.1, seed=1)
    assert Y.shape == H.shape == X.shape and rstd.shape == (0,)
    dX, dR, dw = xb.xconv_rmsnorm_backward(X, X, rstd, w, p=0.1, seed=1)
    assert dX.shape == X.shape and bool((dw == 0).all()) and dw.shape == (40,)
    assert xb.xconv_dropout(X, 0.5, 1).shape == X.shape
    Q, scales, _, _ = xb.xconv_rmsnorm_quantized(X, w, group=32)
    assert xb.xconv_dequantize(Q, scales, group=32).shape == X.shape and scales.shape == (0, 2)
    image = torch.empty(0, 40, 3, 3, device="cuda").contiguous(memory_format=torch.channels_last)
    assert xb.xconv_dropout(image, 0.5, 1, channels=True).shape == image.shape
    # the library's own calls
    d = xb.RowsDesc(rows=0, C=40, dtype=xb.XCONV_BF16, rows_per_mask=1, x_stride=40, r_stride=40, h_stride=40, y_stride=40)
    dw = torch.full((40,), 3.0, device="cuda")
    ws = torch.empty(xb.lib().xconv_rmsnorm_workspace_bytes(ctypes.byref(d)), dtype=torch.uint8, device="cuda")
    p = dw.data_ptr()
    assert xb.lib().xconv_rmsnorm_backward(ctypes.byref(d), p, p, p, None, None, p, None, p, ws.data_ptr(), ws.numel(), None) == 0
    torch.cuda.synchronize()
    assert bool((dw == 0).all())


@pytest.mark.parametrize("C,gap", [(64, 8), (64, 3), (97, 15), (20000, 4)])
def test_nothing_is_written_between_the_rows(C, gap):
    """The library's calls with strided outputs: what lies between the rows and behind the last one stays.  (Strided rows may get their sums in another order than dense ones: the results are
    held to the formulas, as everywhere.)"""
    rows, wide, t = 13, C + gap, torch.bfloat16
    X, res = tensor((rows, C), t, 1), tensor((rows, C), t, 2)
    fresh = lambda dtype=torch.bfloat16: torch.full((rows + 2, wide), 7, device="cuda", dtype=dtype)
    outside = lambda t: bool((t[rows:] == 7).all()) and bool((t[:, C:] == 7).all())
    d = xb.RowsDesc(rows=rows, C=C, dtype=xb.XCONV_BF16, eps=1e-5, x_stride=C, r_stride=C, h_stride=wide, dh_stride=C, y_stride=wide, p=0.25, seed=9, rows_per_mask=1)
    call = lambda name, *a: xb._check(getattr(xb.lib(), name)(ctypes.byref(d), *[t.data_ptr() if isinstance(t, torch.Tensor) else t for t in a], xb._stream()), name)
    Y, H, rstd = fresh(), fresh(), torch.full((rows + 2,), 7.0, device="cuda")
    call("xconv_rmsnorm_forward", X, res, None, H, Y, None, rstd)
    (y, h, s), (y_off, h_off, s_off) = R.norm(X, None, res, 1e-5, 0.25, 9)
    R.close("Y", R.last(Y[:rows, :C]), y, R.rounded(y, y_off, t))
    R.close("H", R.last(H[:rows, :C]), h, R.rounded(h, h_off, t))
    R.close("rstd", rstd[:rows].cpu().double(), s, s_off + 2.0 ** -23 * s)
    assert outside(Y) and outside(H) and bool((rstd[rows:] == 7).all())
    drop = fresh()
    call("xconv_dropout", X, res, drop)
    R.close("dropout", R.last(drop[:rows, :C]), h, R.rounded(h, h_off, t))
    assert outside(drop)
    d.q_type, d.q_group = xb.XCONV_Q_INT8, 32
    Q, scales, again = fresh(torch.int8), torch.full((rows * -(-C // 32) + 5,), 7.0, device="cuda"), fresh()
    call("xconv_rmsnorm_forward", X, res, None, again, Q, scales, rstd)
    check_8_bits(Q[:rows, :C], scales[:-5].view(rows, -1), y, y_off, 32, 127.0)
    assert outside(Q) and outside(again) and bool((scales[-5:] == 7).all())
    d.x_stride = wide
    V = fresh()
    call("xconv_dequantize", Q, scales, V)
    want = R.last(Q[:rows, :C].float()) * R.last(scales[:-5].view(rows, -1)).repeat_interleave(32, 1)[:, :C]
    R.close("V", R.last(V[:rows, :C]), want, R.rounded(want, 0 * want, t))
    assert outside(V)
    d.r_stride = wide
    dX, dR, dw = fresh(), fresh(), torch.full((C + 8,), 7.0, device="cuda")
    ws = torch.empty(xb.lib().xconv_rmsnorm_workspace_bytes(ctypes.byref(d)), dtype=torch.uint8, device="cuda")
    call("xconv_rmsnorm_backward", Y, H, rstd, None, res, dX, dR, dw, ws, ws.numel())
    (dx, dr, dweight), (x_off, r_off, w_off) = R.norm_backward(Y[:rows, :C], H[:rows, :C], rstd[:rows], None, res, 0.25, 9)
    R.close("dX", R.last(dX[:rows, :C]), dx, R.rounded(dx, x_off, t))
    R.close("dresidual", R.last(dR[:rows, :C]), dr, R.rounded(dr, r_off, t))
    R.close("dweight", dw[:C].cpu().double(), dweight, w_off)
    assert outside(dX) and outside(dR) and bool((dw[C:] == 7).all())


def test_gradients_against_differences():
    """Of sum(Y a) + sum(H b) by the forward call's own arithmetic in float, differences of 2^-6 to both sides.  They are off by 2^-12 / 6 of the third derivative (some tens)
    and by the rounding of 120 values of a few units, 2^-20 at most together, over 2^-5."""
    shape = (5, 24)
    X, res, w = tensor(shape, torch.float32, 1), tensor(shape, torch.float32, 2), tensor((24,), torch.float32, 3)
    a, b = tensor(shape, torch.float32, 4), tensor(shape, torch.float32, 5)

    def loss(X, res, w):
        Y, H, _ = xb.xconv_rmsnorm(X, w, residual=res, p=0.4, seed=11)
        return float((Y.double() * a).sum() + (H.double() * b).sum())

    _, H, rstd = xb.xconv_rmsnorm(X, w, residual=res, p=0.4, seed=11)
    dX, dR, dw = xb.xconv_rmsnorm_backward(a, H, rstd, w, dH=b, p=0.4, seed=11)
    for name, t, grad in (("X", X, dX), ("residual", res, dR), ("weight", w, dw)):
        flat, step = t.view(-1), 2.0 ** -6
        for i in range(flat.numel()):
            old = float(flat[i])
            flat[i] = old + step; up = loss(X, res, w); top = float(flat[i])
            flat[i] = old - step; down = loss(X, res, w); width = top - float(flat[i])
            flat[i] = old
            assert abs((up - down) / width - float(grad.view(-1)[i])) < 2e-2, (name, i)


def test_a_block_as_it_is_used():
    """Convolution, dropout, residual and norm of images, forward and backward, against autograd in 64 bits with the same mask; then in 8 bits into the next convolution."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").contiguous(memory_format=torch.channels_last)
    X, W, Z = rnd(4, 24, 10, 9), rnd(24, 24, 3, 3).mul_(0.07).contiguous(memory_format=torch.channels_last), rnd(8, 24, 10, 9)
    g = torch.randn(24, generator=gen, device="cuda")
    dY = rnd(4, 24, 10, 9)
    C, _ = xb.xconv_forward(X, W, Z)
    Y, H, rstd = xb.xconv_rmsnorm(C, g, residual=X, p=0.2, seed=SEED)
    dC, dres, dg = xb.xconv_rmsnorm_backward(dY, H, rstd, g, p=0.2, seed=SEED)
    dX = xb.xconv_dgrad(dC, W) + dres
    x, w, gg = X.double().cpu().requires_grad_(), W.double().cpu(), g.double().cpu().requires_grad_()
    mask = R.kept(4 * 90, 24, 0.2, SEED).view(4, 10, 9, 24).permute(0, 3, 1, 2).double() / 0.8
    h = torch.nn.functional.conv2d(x, w, padding=1) * mask + x
    y = h * (h.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gg.view(1, -1, 1, 1)
    y.backward(dY.double().cpu())
    rel = lambda a, b: float((a.detach().double().cpu() - b.detach()).norm() / b.detach().norm())
    # a few hundred roundings of 2^-24 a value, of independent sign
    assert rel(Y, y) < 2e-6 and rel(dX, x.grad) < 2e-6 and rel(dg, gg.grad) < 2e-6
    Q, scales, H8, _ = xb.xconv_rmsnorm_quantized(C, g, residual=X, p=0.2, seed=SEED)
    assert torch.equal(H8, H)
    Y2, _ = xb.xconv_forward(xb.xconv_dequantize(Q, scales, dtype=torch.float32), W, Z)
    want = torch.nn.functional.conv2d(y.detach(), w, padding=1)
    # (a step of 2^-3 of a value, evenly spread: 2^-4 / sqrt(3) of it at most, and sums keep the relation)
    assert rel(Y2, want) < 2.0 ** -4


@pytest.mark.parametrize("dtype", list(T))
def test_rows_that_are_one_row_and_weights_at_any_address(dtype):
    """A row that is broadcast to all (stride 0), and weights that do not begin on a boundary."""
    t = T[dtype]
    for C in (8, 40, 97, 1024):
        X = tensor((1, C), t, 1, scale=2.0).expand(33, C)
        res = tensor((33, C), t, 2)
        w = tensor((C + 1,), t, 3)[1:]
        Y, H, rstd = xb.xconv_rmsnorm(X, w, residual=res, p=0.3, seed=SEED)
        (y, h, s), (y_off, h_off, _) = R.norm(X, w, res, 1e-6, 0.3, SEED)
        R.close("Y", R.last(Y), y, R.rounded(y, y_off, t))
        R.close("H", R.last(H), h, R.rounded(h, h_off, t))
        dX, dR, dw = xb.xconv_rmsnorm_backward(X, H, rstd, w, dH=X, p=0.3, seed=SEED)
        (dx, dr, dweight), (x_off, r_off, w_off) = R.norm_backward(X, H, rstd, w, X, 0.3, SEED)
        R.close("dX", R.last(dX), dx, R.rounded(dx, x_off, t))
        R.close("dresidual", R.last(dR), dr, R.rounded(dr, r_off, t))
        R.close("dweight", dw.cpu().double(), dweight, w_off + 2.0 ** -24 * dweight.abs())
        D = xb.xconv_dropout(X, 0.3, SEED, residual=res)
        R.close("D", R.last(D), h, R.rounded(h, h_off, t))


def test_two_graphs_and_two_threads():
    """Gradients of two sizes in two captured graphs that are replayed together, and from two host threads: each has scratch memory of its own."""
    import threading
    sets = []
    for rows, C in ((3000, 1024), (2000, 97)):
        H, dY = tensor((rows, C), torch.bfloat16, 1), tensor((rows, C), torch.bfloat16, 2)
        _, _, rstd = xb.xconv_rmsnorm(H)
        sets.append((dY, H, rstd, xb.xconv_rmsnorm_backward(dY, H, rstd)))
    torch.cuda.synchronize()
    graphs = []
    for dY, H, rstd, _ in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = xb.xconv_rmsnorm_backward(dY, H, rstd)
        graphs.append((g, out, torch.cuda.Stream()))
    for _ in range(10):
        for g, _, stream in graphs:
            with torch.cuda.stream(stream):
                g.replay()
    torch.cuda.synchronize()
    for (_, _, _, want), (_, out, _) in zip(sets, graphs):
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    bad = []

    def work(dY, H, rstd, want):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(50):
                got = xb.xconv_rmsnorm_backward(dY, H, rstd)
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    bad.append(1)

    threads = [threading.Thread(target=work, args=s) for s in sets]
    [t.start() for t in threads]; [t.join() for t in threads]
    assert not bad


def test_calls_on_two_streams():
    X, dY, w = tensor((512, 1024), torch.bfloat16, 1), tensor((512, 1024), torch.bfloat16, 2), tensor((1024,), torch.float32, 3)
    _, H, rstd = xb.xconv_rmsnorm(X, w)
    want = xb.xconv_rmsnorm_backward(dY, H, rstd, w)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(xb.xconv_rmsnorm_backward(dY, H, rstd, w))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_the_python_path_gives_the_same_bits(monkeypatch):
    X, res, w = tensor((3, 40, 6, 5), torch.float16, 1), tensor((3, 40, 6, 5), torch.float16, 2), tensor((40,), torch.float16, 3)

    def all_of_them():
        Y, H, rstd = xb.xconv_rmsnorm(X, w, residual=res, p=0.3, seed=4, channels=True)
        Q, scales, _, _ = xb.xconv_rmsnorm_quantized(X, w, residual=res, group=32, p=0.3, seed=4)
        return [Y, H, rstd, *xb.xconv_rmsnorm_backward(res, H, rstd, w, dH=X, p=0.3, seed=4, channels=True), Q.view(torch.uint8), scales, xb.xconv_dequantize(Q, scales, group=32),
                xb.xconv_dropout(X, 0.5, 8, residual=res, channels=True), xb.xconv_dropout(X, 0.5, 8)]

    native = all_of_them()
    monkeypatch.setattr(xb, "_native", xb._Declines())
    for a, b in zip(native, all_of_them()):
        assert torch.equal(a, b) and a.stride() == b.stride() and a.dtype == b.dtype
