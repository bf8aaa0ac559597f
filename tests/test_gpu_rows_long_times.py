"""Long rows that a block's registers hold are read once; beyond them they are read again for every step.  The first form must not be the slower one."""
import pytest
import torch

from paper_2106_06998_b200 import binding as xb
from tests._util import device_time

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("p", [0.0, 0.1])
@pytest.mark.parametrize("C", [8200, 12288, 16384])
def test_gradients_of_long_rows(C, p):
    """A value's time, against that of rows of 16392 values, the shortest that are read again (half of it; where what a thread keeps lies in local memory twice to four times as much)."""
    def time_of(C):
        X, D = (torch.randn(2048, C, device="cuda").to(torch.bfloat16) for _ in range(2))
        w = torch.ones(C, device="cuda")
        _, H, rstd = xb.xconv_rmsnorm(X, w)
        return device_time(lambda: xb.xconv_rmsnorm_backward(D, H, rstd, w, dH=X, p=p, seed=3), calls=10) / C
    assert time_of(C) < 1.05 * time_of(16392)
