"""The largest matrices of a sequence model in 16 bits, where the tensor cores' chains of sums are longest, against the recurrence in 64 bits; and the same bits again
whatever the scratch memory held.

The error allowed is that of test_gpu_update.py, four times the error of the same recurrence in float arithmetic, and the rounding.  For one element it is taken
row by row: the bound there, eight times the root mean square over all elements, holds where all errors are of one size.  Rows of the "few" kind differ by factors of up to
e^4 and their errors with them: float arithmetic itself is off by up to 9.4e-4 of the result's root mean square there (4096 x 1024, float16), where 8 * 4 * 1.77e-5
are 5.7e-4."""
import pytest
import torch

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb
from tests.test_gpu_update import COEFFICIENTS, HALF, TINY, U, check_muon, make, recurrence

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    torch.cuda.set_device(0)


def check(O, G):
    """|error| <= rounding + allowed, over all of the matrix and, with a factor of eight (the largest of ten million normal errors is 5.4 of them), element by element."""
    want = recurrence(G[None].double(), 5, COEFFICIENTS, 1e-7)[0]
    plain = recurrence(G[None].float(), 5, COEFFICIENTS, 1e-7)[0].double() - want
    half, err = HALF[O.dtype], (O.double() - want).abs()
    size = want.square().mean(1, keepdim=True).sqrt()
    allowed = 4 * torch.maximum(plain.square().mean(1, keepdim=True).sqrt(), 16 * U * size)
    assert (err <= (half + 8 * U) * want.abs() + 8 * allowed * (1 + half) + TINY[O.dtype]).all(), float((err / (half * want.abs() + 8 * allowed)).max())
    whole = (half * want.norm() + allowed.square().sum().mul(want.shape[1]).sqrt() * (1 + half) + TINY[O.dtype] * want.numel() ** 0.5)
    assert err.norm() <= whole


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(4096, 4096), (4096, 1024), (1000, 4097)])
def test_orthogonalize(shape, dtype):
    for kind in ("normal", "few"):
        G = make(shape, dtype, seed=11, kind=kind)
        O = xb.xconv_orthogonalize(G)
        check(O, G)
        for fill in (0, 255, 127):         # zeros, NaN of either kind of float
            xb.workspace(1, G.device).fill_(fill)
            assert torch.equal(xb.xconv_orthogonalize(G), O)


def test_the_rounding_to_16_bits_is_nearly_all_of_the_error():
    """The sums' error d moves a result across the border between two roundings, a step s apart, with a probability of |d| / s, and what differs is then s; where |d| is beyond s
    at most |d| + s.  So the squares of the differences from the rounded exact result come to 3 |d| s + d^2 at most, added up to 3 |d| |s| + |d|^2 of the norms.  |d|: four times that
    of float arithmetic, as everywhere; s: at most 2^-7 of the value."""
    G = make((4096, 4096), torch.bfloat16, seed=12, kind="few")
    O = xb.xconv_orthogonalize(G).double()
    want = recurrence(G[None].double(), 5, COEFFICIENTS, 1e-7)[0]
    d = 4 * (recurrence(G[None].float(), 5, COEFFICIENTS, 1e-7)[0].double() - want).norm()
    assert (O - want.bfloat16().double()).square().sum() <= 3 * d * 2.0 ** -7 * want.norm() + d * d


def test_muon_step():
    shapes = [(1024, 1024), (4096, 1024), (1024, 4096)]
    check_muon([make(s, torch.bfloat16, i, scale=0.05) for i, s in enumerate(shapes)], [make(s, seed=i + 10) for i, s in enumerate(shapes)],
               [make(s, seed=i + 20) for i, s in enumerate(shapes)])
