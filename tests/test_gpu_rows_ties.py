"""Values that lie at the same distance from two 8-bit codes go to the even one, in every form of the kernel: codes against whole numbers, without a tolerance."""
import pytest
import torch

from paper_2106_06998_b200 import binding as xb
from tests import _rows as R
from tests.test_gpu_rows import T

pytestmark = pytest.mark.gpu


def whole_numbers(shape, dtype, kind, seed, most):
    """Whole numbers of up to `most` in magnitude: "dense", or some channels of wider rows that begin on an odd one ("cut")."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    extra, first = (5, 3) if kind == "cut" else (0, 0)
    return torch.randint(-most, most + 1, (shape[0], shape[1] + extra), generator=gen, device="cuda").to(dtype)[:, first:first + shape[1]]


def nearest(t, a, M):
    """The codes nearest to t / a (whole numbers, |t| <= M a): of two at the same distance the even one, and how many are such.  By products of whole numbers alone."""
    if M == 448:
        values = torch.tensor([(8 + i % 8) << (i // 8) if i >= 8 else 2 * i for i in range(127)])          # times 2^10
    else:
        values = torch.arange(128) << 10
    borders = (values[1:] + values[:-1]) // 2
    t10 = t.abs() << 10
    code, ties = torch.zeros_like(t), torch.zeros_like(t, dtype=torch.bool)
    for i, b in enumerate(borders.tolist()):
        above = t10 - a * b
        code += ((above > 0) | ((above == 0) & (i % 2 == 1))).long()
        ties |= above == 0
    return torch.where(t < 0, -values[code], values[code]).double() / 1024, int(ties.sum())


# h is 62 at most and 16 times the weight 24: products of up to 11 bits, which are exact, and quotients (times M, less than 9 bits) that are 2^-20 of themselves from every border that they
# do not lie on, farther than their roundings.
@pytest.mark.parametrize("shape,kind", [((300, 64), "dense"), ((300, 4096), "dense"), ((60, 8200), "dense"), ((20, 16640), "dense"), ((3000, 97), "dense"), ((400, 513), "dense"), ((300, 200), "cut"),
                                        ((60, 4100), "cut"), ((20, 9001), "cut")])
@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("q,M", [(torch.float8_e4m3fn, 448), (torch.int8, 127)])
@pytest.mark.parametrize("group", [0, 32, 128])
def test_ties_go_to_the_even_code(shape, kind, dtype, q, M, group):
    t, C = T[dtype], shape[1]
    X, residual = whole_numbers(shape, t, kind, 1, 31), whole_numbers(shape, t, kind, 2, 31)
    weight = torch.randint(8, 25, (C,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(t) / 16
    Q, scales, H, rstd = xb.xconv_rmsnorm_quantized(X, weight, residual=residual, qdtype=q, group=group)
    u = (R.last(X) + R.last(residual)).long() * (weight.cpu().double() * 16).long()
    width = group if 0 < group < C else C
    most = torch.nn.functional.pad(u, (0, -C % width)).reshape(shape[0], -1, width).abs().amax(-1).clamp(min=1).repeat_interleave(width, 1)[:, :C]
    want, ties = nearest(u * M, most, M)
    got = R.last(Q.float())
    assert ties > 0
    assert torch.equal(got, want), f"{int((got != want).sum())} of {got.numel()} codes, where {ties} values are ties"
