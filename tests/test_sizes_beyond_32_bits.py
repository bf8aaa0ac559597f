"""Sizes that do not fit the descriptors' fields of 32 bits are refused by the binding, not cut off (no GPU: tensors without memory)."""
import pytest
import torch

from paper_2106_06998_b200 import binding as xb

B32 = 1 << 32


class _Cuda(torch.Tensor):
    """A tensor without memory that says that it is on the GPU: its layout is looked at before anything is launched."""
    is_cuda = True


def _meta(*shape):
    fmt = {4: torch.channels_last, 5: torch.channels_last_3d}.get(len(shape), torch.contiguous_format)
    return torch.empty(shape, device="meta", memory_format=fmt).as_subclass(_Cuda)


@pytest.mark.parametrize("shape", [(2, B32 + 16), (B32 + 16,), (1, 1 << 31), (1, B32 + 8, 2, 2), (1, B32 + 8, 1, 2, 2)])
def test_rows_of_the_norm(shape):
    with pytest.raises(ValueError, match="does not fit 32 bits"):
        xb._rows(_meta(*shape), "X")


def test_many_rows_and_far_ones_are_no_matter():
    assert xb._rows(_meta(B32 + 16, 3), "X") == ([B32 + 16], 3, 3)
    assert xb._rows(_meta(2, B32 + 16)[:, :24], "X") == ([2], 24, B32 + 16)


@pytest.mark.parametrize("shape", [(4, B32 + 16), (B32 + 16, 4), (B32 + 1, 2, 3), (2, 1 << 31, 1), (2, 1 << 29, 3, 3), (B32 + 3, 1, 1, 1)])
def test_matrices_of_the_update(shape):
    with pytest.raises(ValueError, match="does not fit 32 bits"):
        xb._matrices(_meta(*shape), "G")


@pytest.mark.parametrize("steps", [B32 + 5, -B32 + 5, 1 << 31])
def test_steps_of_the_update(steps):
    t = torch.zeros(4, 8)
    for call in (lambda: xb.xconv_orthogonalize(t, steps=steps), lambda: xb.xconv_muon_step(t, t, t, 0.1, steps=steps)):
        with pytest.raises(ValueError, match="steps = .* does not fit 32 bits"):
            call()
