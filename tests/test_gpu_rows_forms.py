"""Forms of the kernels between the blocks that other tests do not reach, against the formulas in 64 bits: long odd rows by runs, whole channels dropped in front of the norm, seeds in device memory,
8 bits behind a dropout, blocks that take several rows, calls that are large enough for several octets a thread."""
import pytest
import torch

from paper_2106_06998_b200 import binding as xb
from tests import _rows as R
from tests.test_gpu_rows import SEED, T, _seed_tensor, check_8_bits, tensor

pytestmark = pytest.mark.gpu


def channels_of(shape):
    return shape[1] if len(shape) >= 4 else shape[-1]


def norm_and_gradients(X, residual, w, dH, dY, p, seed, channels=False, device_seed=False):
    """Both passes with everything that they can take, held to the formulas."""
    t = X.dtype
    drop = dict(p=p, seed=_seed_tensor(seed) if device_seed else seed, channels=channels)
    Y, H, rstd = xb.xconv_rmsnorm(X, w, residual=residual, eps=1e-5, **drop)
    (y, h, s), (y_off, h_off, s_off) = R.norm(X, w, residual, 1e-5, p, seed, channels)
    R.close("Y", R.last(Y), y, R.rounded(y, y_off, t))
    R.close("H", R.last(H), h, R.rounded(h, h_off, t))
    R.close("rstd", rstd.cpu().double().reshape(-1), s, s_off + 2.0 ** -23 * s)
    dX, dR, dw = xb.xconv_rmsnorm_backward(dY, H, rstd, w, dH=dH, **drop)
    (dx, dr, dweight), (x_off, r_off, w_off) = R.norm_backward(dY, H, rstd, w, dH, p, seed, channels)
    R.close("dX", R.last(dX), dx, R.rounded(dx, x_off, t))
    R.close("dresidual", R.last(dR), dr, R.rounded(dr, r_off, t))
    R.close("dweight", dw.cpu().double(), dweight, w_off + 2.0 ** -24 * dweight.abs())


def both_passes(shape, t, kind, p, **kw):
    X, residual, dY = tensor(shape, t, 1, kind), tensor(shape, t, 2, kind, 3.0), tensor(shape, t, 4, kind)
    norm_and_gradients(X, residual, tensor((channels_of(shape),), t, 3), tensor(shape, t, 5, kind), dY, p, SEED, **kw)


# (4097 and 8191: a block a row, several warps, every block several rows; 513 and 777 the same with two to five warps; 129 and 300: a warp a row)
@pytest.mark.parametrize("shape", [(3000, 129), (900, 300), (5000, 513), (3000, 777), (1300, 4097), (500, 8191), (3, 8191), (1, 2049), (2, 513), (700, 2050)])
@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_long_odd_rows(shape, dtype, p):
    both_passes(shape, T[dtype], "dense", p)


@pytest.mark.parametrize("shape", [(5, 7), (33, 129), (40, 2057), (3, 8203), (2, 16385), (2, 40001), (257, 31), (3, 97, 9, 11), (2, 21, 3, 4, 5), (4, 6, 73)])
@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("q", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("group", [0, 64])
def test_8_bits_of_dense_odd_rows_behind_a_dropout(shape, dtype, q, group):
    in_8_bits(shape, T[dtype], "dense", q, group, 0.3)


def in_8_bits(shape, t, kind, q, group, p, channels=False):
    C = channels_of(shape)
    X, residual, weight = tensor(shape, t, 1, kind), tensor(shape, t, 2, kind, 3.0), tensor((C,), t, 3)
    Q, scales, H, rstd = xb.xconv_rmsnorm_quantized(X, weight, residual=residual, eps=1e-5, qdtype=q, group=group, p=p, seed=SEED, channels=channels)
    (y, h, s), (y_off, h_off, s_off) = R.norm(X, weight, residual, 1e-5, p, SEED, channels)
    R.close("H", R.last(H), h, R.rounded(h, h_off, t))
    R.close("rstd", rstd.cpu().double().reshape(-1), s, s_off + 2.0 ** -23 * s)
    codes, wide = check_8_bits(Q, scales, y, y_off, group if 0 < group < C else C, 448.0 if q == torch.float8_e4m3fn else 127.0)
    V = xb.xconv_dequantize(Q, scales, group=group, dtype=t)
    R.close("V", R.last(V), codes * wide, R.rounded(codes * wide, 0 * wide, t))


@pytest.mark.parametrize("shape,kind", [((1200, 4096), "dense"), ((5000, 72), "dense"), ((9, 8192), "wide"), ((257, 40), "cut"), ((300, 4097), "dense"), ((600, 8200), "dense"), ((500, 12288), "wide"),
                                        ((4, 64, 17, 5), "dense"), ((2, 20000), "shifted")])
@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("q,group,p", [(torch.float8_e4m3fn, 128, 0.1), (torch.int8, 32, 0.3), (torch.float8_e4m3fn, 0, 0.5), (torch.int8, 0, 0.0)])
def test_8_bits_of_many_rows(shape, kind, dtype, q, group, p):
    in_8_bits(shape, T[dtype], kind, q, group, p, channels=len(shape) > 2)


CHANNELS = [(3, 97, 9, 11), (2, 16, 5, 7), (6, 64, 7, 5), (2, 20, 3, 4, 5), (3, 513, 6, 5), (5, 40, 129), (5, 41, 136), (3, 40, 777), (2, 3, 8200), (2, 2, 20001), (1, 96, 40, 40), (70, 25, 1, 1)]


@pytest.mark.parametrize("shape", CHANNELS)
@pytest.mark.parametrize("kind", ["dense", "cut", "wide", "shifted"])
@pytest.mark.parametrize("dtype", list(T))
def test_whole_channels_in_front_of_the_norm(shape, kind, dtype):
    both_passes(shape, T[dtype], kind, 0.3, channels=True)


@pytest.mark.parametrize("shape,kind", [((50, 97), "dense"), ((50, 97), "shifted"), ((300, 513), "dense"), ((20, 4097), "dense"), ((50, 200), "cut"), ((50, 200), "wide"), ((3, 20000), "dense"), ((3, 20001), "dense"),
                                        ((5, 8200), "dense"), ((2, 40, 6, 5), "dense"), ((2, 41, 6, 5), "dense")])
@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("channels", [False, True])
def test_a_seed_in_device_memory_in_every_form(shape, kind, dtype, channels):
    t = T[dtype]
    both_passes(shape, t, kind, 0.3, channels=channels, device_seed=True)
    X, residual = tensor(shape, t, 1, kind), tensor(shape, t, 2, kind, 3.0)
    want = R.dropped(R.last(X), 0.3, SEED, R.per_of(X, channels))
    off = 2.0 ** -22 * (want.abs() + R.last(residual).abs())
    R.close("dropout", R.last(xb.xconv_dropout(X, 0.3, _seed_tensor(SEED), residual=residual, channels=channels)), want + R.last(residual), R.rounded(want + R.last(residual), off, t))


@pytest.mark.parametrize("shape,kind,dtype", [((1200, 4096), "dense", "bf16"), ((1200, 4096), "dense", "f16"), ((1200, 4096), "dense", "f32"), ((1200, 4096), "wide", "bf16"), ((2400, 2052), "dense", "f32"),
                                              ((4, 300, 4096), "dense", "f16"), ((9, 64, 100, 91), "dense", "bf16"), ((9, 64, 100, 91), "dense", "f32")])
@pytest.mark.parametrize("channels", [False, True])
def test_dropout_of_several_octets_a_thread(shape, kind, dtype, channels):
    """(more than 606208 octets of aligned rows)"""
    t = T[dtype]
    X, residual = tensor(shape, t, 1, kind), tensor(shape, t, 2, kind, 3.0)
    assert X.numel() // channels_of(shape) * -(-channels_of(shape) // 8) > 606208
    want = R.dropped(R.last(X), 0.2, SEED, R.per_of(X, channels))
    R.close("Y", R.last(xb.xconv_dropout(X, 0.2, SEED, channels=channels)), want, R.rounded(want, 2.0 ** -23 * want.abs(), t))
    off = 2.0 ** -22 * (want.abs() + R.last(residual).abs())
    want = want + R.last(residual)
    for seed in (SEED, _seed_tensor(SEED)):
        R.close("Y", R.last(xb.xconv_dropout(X, 0.2, seed, residual=residual, channels=channels)), want, R.rounded(want, off, t))
    both = R.last(X) + R.last(residual)
    R.close("sum", R.last(xb.xconv_dropout(X, 0.0, None, residual=residual)), both, R.rounded(both, 2.0 ** -23 * both.abs(), t))


# 16-bit rows of four octets a thread, floats that are read again: blocks that take several rows.
@pytest.mark.parametrize("shape,dtype", [((1900, 8200), "bf16"), ((1900, 8200), "f16"), ((700, 16384), "bf16"), ((700, 16384), "f16"), ((1300, 8200), "f32"), ((700, 16392), "bf16")])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_blocks_that_take_several_long_rows(shape, dtype, p):
    both_passes(shape, T[dtype], "dense", p)
