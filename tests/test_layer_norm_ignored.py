"""Fields of the norm's descriptor that a call does not look at (no GPU: nothing is launched)."""
import ctypes

import pytest

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb


@pytest.mark.parametrize("dx_stride", [-1, -2 ** 63, 1 << 61, 2 ** 63 - 1, 0])
def test_the_forward_call_does_not_look_at_dx_stride(dx_stride):
    """A call with a misaligned output comes past the descriptor's checks and is refused behind them; the gradients and their scratch memory refuse the stride."""
    entry.build()
    L = xb.lib()
    desc = xb.NormDesc(6, 40, xb.XCONV_BF16, xb.XCONV_F32, 1e-5, 40, 40, dx_stride)
    assert L.xconv_layernorm_forward(ctypes.byref(desc), 16, None, None, 17, None, None, None) == 3
    want = 1 if dx_stride <= 0 else 2
    assert L.xconv_layernorm_backward(ctypes.byref(desc), 16, 16, 16, 16, None, 16, 16, 16, 16, 1 << 30, None) == want
    if dx_stride:
        assert L.xconv_layernorm_workspace_bytes(ctypes.byref(desc)) == 0
