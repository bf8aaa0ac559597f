"""Batches that go through the scratch memory in several parts: a part begins at any matrix of the batch, on any boundary.  The sizes here are those where that boundary
is not one of 16 bytes, which the first test shows by the library's own arithmetic (restated; no GPU)."""
import pytest
import torch

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb
from tests.test_gpu_update import check, check_muon, make

BLOCKS = 65536                           # of scratch memory that the matrices of a part hold at most


@pytest.fixture(autouse=True)
def _built(request):
    if "gpu" in request.keywords:
        entry.build()
        torch.cuda.set_device(0)


def cuts(shapes):
    """Per tensor: the matrices that a part begins with."""
    out, used, entries = [], 0, 0
    for batch, rows, cols in shapes:     # (the longest sides first)
        n, m = min(rows, cols), max(rows, cols)
        nt = (n + 127) // 128
        each, done, begins = 2 * nt * ((m + 63) // 64) + (2 * nt) ** 2, 0, []
        while done < batch:
            room = max(0, BLOCKS - used) // each
            if entries == 64 or (room == 0 and entries):
                used = entries = 0
                continue
            begins.append(done)
            count = min(max(room, 1), batch - done)
            used, entries, done = used + count * each, entries + 1, done + count
        out.append(begins)
    return out


# 489 matrices in the first part; 14 in it (room for 14 and a half); 38 behind what the other tensor left; two that need more than a part each
CASES = [[(490, 3, 4097)], [(15, 3001, 3001)], [(125, 1024, 1024), (45, 201, 333)], [(2, 16385, 16387)]]


@pytest.mark.parametrize("shapes", CASES)
def test_the_parts_begin_off_the_boundaries(shapes):
    begins = cuts(shapes)[-1]
    _, rows, cols = shapes[-1]
    assert len(begins) == 2 and begins[1] * rows * cols * 4 % 16 and begins[1] * rows * cols * 2 % 8


def around(shapes):
    """Of every tensor: its first and last matrix and those on both sides of a cut."""
    return [sorted({i for c in begins for i in (c - 1, c) if i >= 0} | {0, batch - 1}) for begins, (batch, _, _) in zip(cuts(shapes), shapes)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shapes", CASES[:3])
def test_orthogonalize(shapes, dtype):
    Gs = [make(s, dtype, seed=i) for i, s in enumerate(shapes)]
    for O, G, some in zip(xb.xconv_orthogonalize(Gs), Gs, around(shapes)):
        assert O.isfinite().all()
        check(O[some], G[some])


@pytest.mark.gpu
@pytest.mark.parametrize("gt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shapes", CASES[:3])
def test_muon_step(shapes, gt, monkeypatch):
    """All of the momenta, and the weights of the matrices around the cuts, with those matrices' copies as what the step is checked on."""
    Ws, dWs = [make(s, torch.bfloat16, i, scale=0.05) for i, s in enumerate(shapes)], [make(s, gt, i + 10) for i, s in enumerate(shapes)]
    Ms = [make(s, seed=i + 20) for i, s in enumerate(shapes)]
    some = around(shapes)
    pick = lambda ts: [t[i].clone() for t, i in zip(ts, some)]
    W, dW, M = pick(Ws), pick(dWs), pick(Ms)
    moved = [m + (1 - 0.95) * (g.float() - m) for g, m in zip(dWs, Ms)]
    sizes = [g.float().abs() + m.abs() for g, m in zip(dWs, Ms)]
    xb.xconv_muon_step(Ws, dWs, Ms, 0.02, weight_decay=0.01)
    for m, want, size in zip(Ms, moved, sizes):
        assert ((m - want).abs() <= 8 * 2.0 ** -24 * size).all()          # (three roundings to float on either side, and two factors of 0.05 that may differ)
    got_W, got_M = pick(Ws), pick(Ms)

    def done(w, g, m, *a, **kw):         # (check_muon makes the call itself: here it finds the results of the one above)
        for t, u in zip(w + m, got_W + got_M):
            t.copy_(u)
        return w

    monkeypatch.setattr(xb, "xconv_muon_step", done)
    check_muon(W, dW, M)
