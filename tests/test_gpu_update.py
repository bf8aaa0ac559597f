"""Orthogonalisation by Newton-Schulz products and the step of a network's weights, against their formulas in 64 bits.

The products are said to be as exact as products of floats: two float16 parts hold a value to 2^-24 of it or better, as a float does, the product of two second
parts that is left out is below 2^-24 of the whole, and the sums are rounded like floats' or better.  So the error may be up to four times that of the same recurrence in
float arithmetic on the same input (operands, their second factors, the left out product, sums: each no more than a float's rounding), and where that happens to be
small (a matrix of one value) 64 half steps of a float: five steps of three products whose terms are up to four times their result.  One element may be off by eight
times that (of the root mean square): the largest of a million normal errors is five of them."""
import threading

import pytest
import torch

import __graft_entry__ as entry
from paper_2106_06998_b200 import binding as xb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
FORMAT = {4: torch.channels_last, 5: torch.channels_last_3d}
COEFFICIENTS = xb.NEWTON_SCHULZ
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    torch.cuda.set_device(0)


def matrices(t):
    """(batch, rows, columns): a convolution's rows in the order of memory."""
    return t.movedim(1, -1).reshape(1, t.shape[0], -1) if t.dim() >= 4 else t if t.dim() == 3 else t[None]


def recurrence(G, steps, coefficients, eps):
    X = G.transpose(1, 2) if G.shape[1] > G.shape[2] else G
    X = X / X.double().square().sum((1, 2), keepdim=True).sqrt().clamp(min=eps).to(X.dtype)
    a, b, c = coefficients
    for _ in range(steps):
        A = X @ X.transpose(1, 2)
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.transpose(1, 2) if G.shape[1] > G.shape[2] else X


def bounds(G, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """The orthogonalised matrices in 64 bits, and the error allowed of each, relative to its norm."""
    G = matrices(G)
    want = recurrence(G.double(), steps, coefficients, eps)
    norm = want.square().sum((1, 2)).sqrt()
    plain = (recurrence(G.float(), steps, coefficients, eps).double() - want).square().sum((1, 2)).sqrt()
    return want, 4 * torch.maximum(plain / norm.clamp(min=1e-300), torch.full_like(norm, 16 * U))


def check(O, G, **kw):
    want, tol = bounds(G, **kw)
    half, err = HALF[O.dtype], (matrices(O).double() - want).abs()
    norm = want.square().sum((1, 2)).sqrt()
    rms = (norm / (want.shape[1] * want.shape[2]) ** 0.5)[:, None, None]
    tiny = TINY[O.dtype]
    assert (err.square().sum((1, 2)).sqrt() <= (tol * (1 + half) + half) * norm + tiny * (want.shape[1] * want.shape[2]) ** 0.5).all(), (
        float((err.square().sum((1, 2)).sqrt() / norm).max()), float(tol.max()))
    assert (err <= 8 * tol[:, None, None] * rms * (1 + half) + half * want.abs() + tiny).all()


def make(shape, dtype=torch.float32, seed=0, kind="normal", scale=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    t = rnd(*shape)
    if kind == "few":                      # eight directions above noise, rows of different size
        m = t.reshape(t.shape[0], -1) if t.dim() != 3 else t
        k = min(8, m.shape[-1], m.shape[-2])
        big = rnd(*m.shape[:-1], k) @ rnd(*m.shape[:-2], k, m.shape[-1])
        t = ((0.05 * m + big) * rnd(*m.shape[:-1], 1).exp()).reshape(shape)
    fmt = {4: torch.channels_last, 5: torch.channels_last_3d}.get(len(shape), torch.contiguous_format)
    return (scale * t).to(dtype).contiguous(memory_format=fmt)


SHAPES = [(1, 1), (1, 5), (7, 1), (2, 3), (64, 64), (3, 27), (16, 75), (128, 128), (129, 64), (63, 257), (130, 400), (200, 1000), (1000, 523), (513, 514), (65, 2000),
          (3, 70, 33), (5, 130, 140), (200, 9, 12), (32, 16, 5, 5), (64, 64, 3, 3), (10, 3, 1, 1), (16, 8, 3, 3, 3), (640, 2000), (1, 3000), (3, 1, 300)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize_of_any_shape(shape, dtype):
    for kind in ("normal", "few"):
        G = make(shape, dtype, seed=len(shape) + shape[0], kind=kind)
        before = G.clone()
        O = xb.xconv_orthogonalize(G)
        assert O.shape == G.shape and O.dtype == dtype and O.is_contiguous(memory_format=FORMAT.get(O.dim(), torch.contiguous_format)) and torch.equal(G, before)
        check(O, G)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(16, 193), (17, 192), (32, 191), (32, 1535), (1535, 31), (33, 34), (16, 2), (1, 1000), (5, 15, 1537), (32, 32, 3, 3)])
def test_sides_of_up_to_32(shape, dtype):
    for kind in ("normal", "few"):
        G = make(shape, dtype, seed=5, kind=kind)
        check(xb.xconv_orthogonalize(G), G)


def test_small_sides_beside_larger_ones():
    G = [make(s, seed=k) for k, s in enumerate([(16, 6, 5, 5), (120, 1400), (10, 84), (32, 700), (33, 40), (3, 20, 30)])]
    for O, again, g in zip(xb.xconv_orthogonalize(G), xb.xconv_orthogonalize(G), G):
        check(O, g)
        assert torch.equal(O, again)           # (alone it may be shared among fewer CTAs: sums in another order)


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_any_number_of_steps(steps):
    for shape in ((100, 300), (300, 100), (2, 40, 50)):
        G = make(shape, kind="few")
        check(xb.xconv_orthogonalize(G, steps=steps), G, steps=steps)


def test_steps_that_converge_give_the_orthogonal_factor():
    """a, b, c = 15/8, -10/8, 3/8: every singular value goes to 1, and X X^T to the identity."""
    G = make((96, 200))
    O = xb.xconv_orthogonalize(G, steps=20, coefficients=(1.875, -1.25, 0.375))
    want, tol = bounds(G, steps=20, coefficients=(1.875, -1.25, 0.375))
    P, _, Q = torch.linalg.svd(G.double(), full_matrices=False)
    assert (want[0] - P @ Q).abs().max() < 1e-9
    assert ((O.double() @ O.double().T - torch.eye(96, device="cuda")).square().sum().sqrt() <= 3 * tol * 96 ** 0.5).all()


def test_a_list_of_tensors_is_worked_on_together():
    """More items than one launch takes, of every kind; the same as one call for each, up to the order of sums."""
    shapes = [(64, 64, 3, 3), (1, 9), (16, 3, 5, 5), (130, 260), (2, 33, 70), (300, 40), (8, 8, 3, 3, 3)] * 11
    Gs = [make(s, (torch.float32, torch.bfloat16, torch.float16)[i % 3], seed=i, kind=("normal", "few")[i % 2]) for i, s in enumerate(shapes)]
    Os = xb.xconv_orthogonalize(Gs)
    assert len(Os) == len(Gs) == 77
    for G, O in zip(Gs, Os):
        check(O, G)
    assert xb.xconv_orthogonalize([]) == []


@pytest.mark.parametrize("scale", [1e-37, 1e-20, 1.0, 1e18, 1e36])
def test_gradients_of_any_size(scale):
    """The norm is taken in 64 bits and divided out before anything is rounded to 16 bits; below the smallest normal float (the fourth of these values at 1e-37) the
    input itself has fewer bits, which both sides read."""
    G = make((70, 90), scale=scale)
    check(xb.xconv_orthogonalize(G, eps=0.0), G, eps=0.0)


def test_a_norm_below_eps_and_a_matrix_of_zeros():
    """X = U / eps then.  What is below 2^-38 in X is lost, and grows by no more than 3.4445 a step."""
    Z = torch.zeros((3, 40, 50), device="cuda")
    assert (xb.xconv_orthogonalize(Z) == 0).all()
    G = make((40, 50), scale=1e-9)
    want = recurrence(matrices(G).double(), 5, COEFFICIENTS, 1e-5)
    O = xb.xconv_orthogonalize(G, eps=1e-5)
    lost = 3.4445 ** 5 * 2.0 ** -38 * (40 * 50) ** 0.5
    assert (O.double() - want[0]).square().sum().sqrt() <= lost + 64 * U * want.square().sum().sqrt()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_matrix_that_is_not_finite_is_the_only_one(bad):
    Gs = [make((5, 130, 140), seed=1), make((64, 64, 3, 3), seed=2), make((300, 20), seed=3)]
    fine = xb.xconv_orthogonalize(Gs)
    Gs[0][2, 7, 100] = bad
    Gs[2][299, 19] = bad
    O = xb.xconv_orthogonalize(Gs)
    others = [0, 1, 3, 4]
    assert O[0][2].isnan().all() and O[2].isnan().all()
    assert torch.equal(O[0][others], fine[0][others]) and torch.equal(O[1], fine[1])


def test_more_matrices_than_the_scratch_memory_holds_at_once():
    """600 matrices of 1024 x 1024 go through the kernels some at a time, and come back in order."""
    G = make((600, 1024, 1024), torch.bfloat16, seed=9, scale=1.0)
    O = xb.xconv_orthogonalize(G)
    for i in (0, 1, 127, 128, 255, 256, 599):
        check(O[i], G[i])
    del O


def muon_want(W, dW, M, lr, momentum, nesterov, weight_decay, adjust, **kw):
    g, m = dW.double(), M.double()
    m = m + (1 - momentum) * (g - m)
    u = g + momentum * (m - g) if nesterov else m
    O, tol = bounds(u.float(), **kw)       # (u is rounded to float on its way: the recurrence takes it as it is)
    rows, cols = O.shape[1:]
    s = max(1.0, rows / cols) ** 0.5 if adjust == "spectral" else 0.2 * max(rows, cols) ** 0.5
    w = matrices(W).double()
    return matrices(m), w * (1 - lr * weight_decay) - lr * s * O, tol, abs(lr) * s, O


def check_muon(W, dW, M, lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.01, adjust="spectral", call=None, **kw):
    """M has three roundings to float.  u has five, of sizes up to |g| + |m|: their effect on the orthogonalised matrix is that of an input rounded twice as coarsely
    again (the tolerance's factor 4 becomes 12).  W is rounded to its type once, behind three roundings to float."""
    want = [muon_want(w, g, m, lr, momentum, nesterov, weight_decay, adjust, **kw) for w, g, m in zip(W, dW, M)]
    sizes = [matrices(g).double().abs() + matrices(m).double().abs() for g, m in zip(dW, M)]
    assert xb.xconv_muon_step(W, dW, M, lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, adjust=adjust, **kw) is W
    for w, m, size, (m1, w1, tol, f, O) in zip(W, M, sizes, want):
        assert ((matrices(m).double() - m1).abs() <= 4 * U * size).all()
        norm = O.square().sum((1, 2)).sqrt()
        rms = (norm / (O.shape[1] * O.shape[2]) ** 0.5)[:, None, None]
        tol = 3 * tol[:, None, None]
        err, half = (matrices(w).double() - w1).abs(), HALF[w.dtype]
        assert (err <= (half + 3 * U) * (w1.abs() + f * O.abs()) * (1 + half) + f * 8 * tol * rms + TINY[w.dtype]).all(), float(err.max())
        rounding = ((half + 3 * U) * (w1.abs() + f * O.abs()) + TINY[w.dtype]).square().sum((1, 2)).sqrt()
        assert (err.square().sum((1, 2)).sqrt() <= rounding + f * tol[:, 0, 0] * norm).all()


NETWORK = [(16, 3, 5, 5), (32, 16, 5, 5), (64, 32, 3, 3), (64, 64, 1, 1), (130, 70), (10, 300), (2, 40, 60), (8, 8, 3, 3, 3)]


def network(wt, gt, seed=0):
    W = [make(s, wt, seed=seed + i, scale=0.05) for i, s in enumerate(NETWORK)]
    dW = [make(s, gt, seed=seed + 100 + i, kind=("normal", "few")[i % 2]) for i, s in enumerate(NETWORK)]
    M = [make(s, seed=seed + 200 + i) for i, s in enumerate(NETWORK)]
    return W, dW, M


@pytest.mark.parametrize("wt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("gt", [torch.float32, torch.bfloat16, torch.float16])
def test_muon_step_of_a_network(wt, gt):
    W, dW, M = network(wt, gt)
    check_muon(W, dW, M)
    check_muon(W, network(wt, gt, 50)[1], M)               # and a second one, from the momenta of the first


@pytest.mark.parametrize("kw", [dict(nesterov=False), dict(momentum=0.0), dict(momentum=1.0), dict(weight_decay=0.0, adjust="rms"), dict(lr=0.0), dict(steps=3), dict(lr=-0.1)])
def test_muon_options(kw):
    check_muon(*network(torch.float32, torch.float32), **kw)


def test_muon_step_of_one_tensor():
    W, dW, M = (t[2] for t in network(torch.float32, torch.float32))
    Ws, Ms = [W.clone(memory_format=torch.preserve_format)], [M.clone(memory_format=torch.preserve_format)]
    assert xb.xconv_muon_step(W, dW, M, 0.02, weight_decay=0.01) is W
    check_muon(Ws, [dW], Ms)
    assert torch.equal(W, Ws[0]) and torch.equal(M, Ms[0])


def test_a_training_step_of_a_normed_layer():
    """Norm, convolution and sketch, the estimate, the norm's gradients and the step of the weights, as a program runs them -- eagerly, and captured into a graph
    that is replayed on new inputs."""
    from paper_2106_06998_b200 import inputs
    lay = inputs.make_custom(16, 32, 48, 20, 18, 8, dtype="bf16", seed=3, z="rademacher", x="relu")
    X, W, dY, Z = (xb.to_device(lay[k], "bf16") for k in ("X", "W", "dY", "Z"))
    w, b = torch.ones(32, device="cuda"), torch.zeros(32, device="cuda")
    M = torch.zeros(W.shape, device="cuda").contiguous(memory_format=torch.channels_last)

    def step():
        H, mean, rstd = xb.xconv_layernorm(X, w, b)
        Y, S = xb.xconv_forward(H, W, Z)
        dW = xb.xconv_wgrad(S, dY, Z)
        dH = xb.xconv_dgrad(dY, W)
        dX, dw, db = xb.xconv_layernorm_backward(dH, X, mean, rstd, w)
        xb.xconv_muon_step(W, dW, M, 0.02)
        return H, Y, S, dW, dH, dX, dw, db

    W0 = W.clone(memory_format=torch.preserve_format)
    eager = step()
    W1, M1 = W.clone(memory_format=torch.preserve_format), M.clone(memory_format=torch.preserve_format)
    assert all(t.isfinite().all() for t in eager) and not torch.equal(W0, W1)
    W2, M2 = W0.clone(memory_format=torch.preserve_format), torch.zeros_like(M)
    check_muon([W2], [eager[3]], [M2], weight_decay=0.0)
    assert torch.equal(W2, W1) and torch.equal(M2, M1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    W.copy_(W0); M.zero_()
    graph.replay()
    assert all(torch.equal(g, e) for g, e in zip(captured, eager)) and torch.equal(W, W1) and torch.equal(M, M1)
    X.copy_(X.flip(0)); W.copy_(W0); M.zero_()
    graph.replay()
    W3, M3 = W.clone(memory_format=torch.preserve_format), M.clone(memory_format=torch.preserve_format)
    got = [t.clone() for t in captured]
    W.copy_(W0); M.zero_()
    assert all(torch.equal(g, e) for g, e in zip(got, step())) and torch.equal(W, W3) and torch.equal(M, M3)


def test_the_same_bits_again_on_other_streams():
    Gs = [make(s, seed=i) for i, s in enumerate(NETWORK + [(513, 700), (5, 130, 140)])]
    want = xb.xconv_orthogonalize(Gs)
    torch.cuda.synchronize()
    got, errors = [], []

    def job():
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(10):
                    out = xb.xconv_orthogonalize(Gs)
            s.synchronize()
            got.append(out)
        except Exception as e:
            errors.append(e)

    threads = [threading.Thread(target=job) for _ in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors and len(got) == 4
    assert all(torch.equal(a, b) for out in got for a, b in zip(out, want))


def test_two_captured_graphs_share_no_scratch():
    """Graphs of different sizes, replayed in turn and side by side."""
    Gs = [make((300, 400), seed=1), make((64, 64, 3, 3), seed=2)]
    want = [xb.xconv_orthogonalize(G) for G in Gs]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], []
    for G in Gs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(xb.xconv_orthogonalize(G))
        graphs.append(graph)
        streams.append(torch.cuda.Stream())
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_no_wait_ran_out():
    G = make((513, 700))
    xb.xconv_orthogonalize(G)
    assert xb.workspace_status(xb.workspace(256, G.device)) == 0
