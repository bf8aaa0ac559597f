"""Refusals of the update's entry points and of their binding, sizes of the scratch memory, and the sources' order of starts (no GPU: nothing is launched)."""
import ctypes
import os
import re

import pytest
import torch

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb

UPDATE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2106_06998_b200", "csrc", "update")
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return xb.lib()


def _desc(**kw):
    base = dict(steps=5, a=3.4445, b=-4.775, c=2.0315, eps=1e-7, lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=1, adjust=0)
    base.update(kw)
    return xb.UpdateDesc(**base)


def _item(**kw):
    base = dict(G=16 * MB, M=32 * MB, O=48 * MB, rows=64, cols=576, batch=1, g_dtype=0, o_dtype=0)
    base.update(kw)
    return xb.Matrices(**base)


def _call(fn, desc, items, ws=16, n=1 << 40):
    array = (xb.Matrices * max(1, len(items)))(*items)
    return fn(ctypes.byref(desc) if desc else None, array, len(items), ws, n, None)


def test_refusals_of_the_entry_points(lib):
    for fn in (lib.xconv_orthogonalize, lib.xconv_muon_step):
        assert _call(fn, None, [_item()]) == 1 and fn(ctypes.byref(_desc()), None, 1, 16, 1 << 40, None) == 1 and _call(fn, _desc(), []) == 1
        for kw in (dict(steps=0), dict(steps=-1), dict(steps=65), dict(eps=-1.0), dict(eps=float("nan")), dict(a=float("nan")), dict(c=float("inf"))):
            assert _call(fn, _desc(**kw), [_item()]) == 1, kw
        # a step that takes singular values out of the range in which the operands are held
        for kw in (dict(a=8.0, b=0.0, c=0.0), dict(a=3.4445, b=0.0, c=0.0), dict(a=0.0, b=0.0, c=9.0), dict(a=2.0, b=-10.0, c=0.0)):
            assert _call(fn, _desc(**kw), [_item()]) == 2, kw
        for kw in (dict(G=None), dict(O=None), dict(rows=0), dict(cols=-4), dict(batch=0), dict(g_dtype=3), dict(o_dtype=-1)):
            assert _call(fn, _desc(), [_item(), _item(**{**dict(G=64 * MB, M=80 * MB, O=96 * MB), **kw})]) == 1, kw
        for kw in (dict(G=16 * MB + 8), dict(O=48 * MB + 4)):
            assert _call(fn, _desc(), [_item(**kw)]) == 3, kw
        assert _call(fn, _desc(), [_item(rows=1 << 25)]) == 2 and _call(fn, _desc(), [_item(rows=1 << 18, cols=1 << 18, G=1 << 44, O=1 << 45, M=1 << 46)]) == 2
        need = lib.xconv_update_workspace_bytes((xb.Matrices * 1)(_item()), 1)
        assert need > 0 and _call(fn, _desc(), [_item()], n=need - 1) == 4 and _call(fn, _desc(), [_item()], ws=None) == 4 and _call(fn, _desc(), [_item()], ws=24) == 3
        # what is written overlaps what another item (or the same one) reads or writes
        size = 64 * 576 * 4
        for other in (dict(G=64 * MB, M=80 * MB), dict(G=64 * MB, M=80 * MB, O=48 * MB + size - 16), dict(G=48 * MB + size - 16, M=80 * MB, O=96 * MB),
                      dict(G=64 * MB, M=80 * MB, O=16 * MB), dict(G=96 * MB, M=80 * MB, O=96 * MB)):
            assert _call(fn, _desc(), [_item(), _item(**other)]) == 1, other
    for kw in (dict(lr=float("nan")), dict(momentum=-0.1), dict(momentum=1.5), dict(momentum=float("nan")), dict(weight_decay=float("inf")), dict(nesterov=2), dict(adjust=2)):
        assert _call(lib.xconv_muon_step, _desc(**kw), [_item()]) == 1, kw
    assert _call(lib.xconv_muon_step, _desc(), [_item(M=None)]) == 1 and _call(lib.xconv_muon_step, _desc(), [_item(M=32 * MB + 4)]) == 3
    assert _call(lib.xconv_muon_step, _desc(), [_item(M=48 * MB + 16)]) == 1 and _call(lib.xconv_muon_step, _desc(), [_item(M=16 * MB)]) == 1


def test_scratch_memory_is_bounded(lib):
    size = lambda *items: lib.xconv_update_workspace_bytes((xb.Matrices * len(items))(*items), len(items))
    one = size(_item(rows=300))
    assert one < size(_item(rows=300), _item(rows=300)) < 2 * one + 4096
    assert size(_item()) == 256 and size(_item(), _item(rows=300)) > one      # (small matrices alone lie in shared memory)
    # any number of matrices: 2 GB, and the last one of a table that was not full
    big = _item(rows=1024, cols=1024, batch=100000)
    assert size(big) <= (2 << 30) + (8 << 20) and size(*[big] * 5) == size(big)
    assert size(_item(rows=65536, cols=65536)) > 2 << 30          # a single one takes what it needs
    for kw in (dict(rows=0), dict(batch=-1), dict(rows=1 << 25), dict(rows=1 << 18, cols=1 << 18)):
        assert size(_item(**kw)) == 0, kw


class _Cuda(torch.Tensor):
    """A host tensor that says that it is on the GPU: its layout is looked at before anything is launched."""
    is_cuda = True


def test_the_binding_refuses_what_it_cannot_read(lib):
    fake = lambda t: t.as_subclass(_Cuda)
    with pytest.raises(ValueError):
        xb.xconv_orthogonalize(torch.zeros(4, 8))          # host memory
    for t in (torch.zeros(8, 4).T, torch.zeros(4), torch.zeros(4, 3, 3, 3), torch.zeros(0, 4), torch.zeros(3, 4, 5)[:, :, 1:]):
        with pytest.raises(ValueError):
            xb._matrices(fake(t), "G")
    assert xb._matrices(fake(torch.zeros(4, 8)), "G") == (4, 8, 1) and xb._matrices(fake(torch.zeros(2, 4, 8)), "G") == (4, 8, 2)
    assert xb._matrices(fake(torch.zeros(4, 8, 3, 3).contiguous(memory_format=torch.channels_last)), "G") == (4, 72, 1)
    W = torch.zeros(4, 8)
    for args in (([W, W], [W], [W]), ([W], [W], []), ([W], [torch.zeros(4, 9)], [W])):
        with pytest.raises(ValueError):
            xb.xconv_muon_step(*args, 0.1)
    with pytest.raises(ValueError):
        xb.xconv_muon_step(W, W, W, 0.1, adjust="none")


def test_kernels_that_take_tensor_memory_do_so_before_they_let_the_next_one_start():
    """The rule of the layers' kernels (test_split_sources.py) for those of this folder: one allocation, by one warp, the go-ahead behind it and nowhere else."""
    code = "".join(re.sub(r"//[^\n]*", "", open(os.path.join(UPDATE, f)).read()) for f in sorted(os.listdir(UPDATE)) if f.endswith((".cu", ".cuh")))
    assert code.count("tcgen05.alloc") == 1
    alloc = code.split("void pair_alloc_then_trigger(")[1].split("\n}\n")[0]
    assert alloc.index("tcgen05.alloc") < alloc.index("pdl_trigger()") and alloc.count("pdl_trigger()") == 1
    kernels = [c for c in code.split("\n}\n") if "alloc_then_trigger(&" in c]
    assert len(kernels) == 2 and len(re.findall(r"tmem_alloc|pair_alloc", code)) == 3
    for k in kernels:
        assert re.search(r"if \(warp == [01]\) (pair|tmem)_alloc_then_trigger\(", k) and "pdl_trigger(" not in k and len(re.findall(r"(?:pair|tmem)_dealloc\(", k)) == 1
    assert "__ldg" not in code and "ld.global.nc" not in code      # (what the kernel before writes is not read through the read-only cache)
