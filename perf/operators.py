"""Operators around a layer: layer norm over the channels, forward and backward, and the update of the weights from their gradients (momentum and
orthogonalisation by Newton-Schulz products, as the Muon optimiser does).

A case is one call of an operator:

  norm           Y, mean and rstd of every pixel or token
  norm_backward  dX, dweight, dbias
  orthogonalize  one tensor of gradients: a convolution's weights, a matrix or a batch of matrices
  muon           the step of all weights of a network: weights and momenta in place

Tensors are on the GPU as the library takes them: images channels-last, matrices row-major.  Activations have a mean that differs between the channels
and a few channels that are ten times the others; gradients are a few directions above noise, with rows of different size.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_STEPS, _COEFFICIENTS, _EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
_LR, _MOMENTUM, _DECAY = 0.02, 0.95, 0.01
_NORM_EPS = 1e-5


def _norm(name, op, dtype, B, C, H, W, params="f32"):
    """H = 0: a matrix of B tokens of C values; else a channels-last image batch.  params: the type of weight and bias."""
    return dict(name=name, op=op, dtype=dtype, B=B, C=C, H=H, W=W, params=params)


def listed():
    return [
        # A single token of a decoder, or the pooled vector behind a network's last stage: latency.
        _norm("norm_token_bf16", "norm", "bf16", 1, 4096, 0, 0),
        # The norm in a block of an ImageNet network's middle stage.
        _norm("norm_image_bf16", "norm", "bf16", 64, 128, 56, 56),
        # The last, short batch of an epoch on images of odd size, an odd number of channels: no row is aligned.
        _norm("norm_ragged_f16", "norm", "f16", 50, 97, 35, 27, params="f16"),
        # A small image batch, backward.
        _norm("norm_small_backward_f32", "norm_backward", "f32", 8, 96, 14, 14),
        # Many tokens of a wide model, backward.
        _norm("norm_tokens_backward_bf16", "norm_backward", "bf16", 8192, 4096, 0, 0, params="bf16"),
        # Images of odd size and an odd number of channels, backward.
        _norm("norm_ragged_backward_f16", "norm_backward", "f16", 50, 97, 35, 27),
        # The gradient of one 3 x 3 layer of a small network: latency.
        dict(name="orthogonalize_layer_f32", op="orthogonalize", dtype="f32", shape="64:64:3:3"),
        # A batch of matrices of odd sizes, taller than wide (expert or per-group weights), half precision.
        dict(name="orthogonalize_batch_f16", op="orthogonalize", dtype="f16", shape="8:1000:523"),
        # A square projection of a wide model: the largest case.
        dict(name="orthogonalize_wide_bf16", op="orthogonalize", dtype="bf16", shape="4096:4096"),
        # All layers of the CIFAR-10 network with 5 x 5 kernels.
        dict(name="muon_cifar_f32", op="muon", dtype="f32", layers="16:3:5:5 32:16:5:5 32:32:5:5"),
        # All convolutions of a residual network for ImageNet.
        dict(name="muon_resnet_f32", op="muon", dtype="f32",
             layers="64:64:3:3*4 128:64:3:3 128:128:3:3*3 256:128:3:3 256:256:3:3*3 512:256:3:3 512:512:3:3*3 128:64:1:1 256:128:1:1 512:256:1:1"),
        # Two blocks of a sequence model, weights in bfloat16.
        dict(name="muon_blocks_bf16", op="muon", dtype="bf16", layers="1024:1024*8 4096:1024*2 1024:4096*2"),
    ]


def _shape(text):
    return tuple(int(v) for v in text.split(":"))


def _layers(text):
    out = []
    for item in text.split():
        shape, _, times = item.partition("*")
        out += [_shape(shape)] * int(times or 1)
    return out


def _matrices(shape):
    """(batch, rows, columns) of a tensor: matrices and batches of them as they are, weights of a convolution one row per output channel."""
    if len(shape) == 3:
        return shape
    return 1, shape[0], math.prod(shape[1:])


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of the same ranges.  Norms: 8 to 8192 channels, on and off the multiples of 8, one row up to the elements of the largest listed case.
    Orthogonalisation: matrices of 1 to 4096 rows and columns, convolutions, batches.  Steps: up to 24 layers of one network."""
    flops_max = max(work(c)["flops"] for c in listed())
    while True:
        op = rng.choice(["norm"] * 3 + ["norm_backward"] * 4 + ["orthogonalize"] * 3 + ["muon"] * 3)
        dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
        if op in ("norm", "norm_backward"):
            C = _log_int(rng, 8, 8192) if rng.random() < 0.4 else 8 * _log_int(rng, 1, 1024)
            rows_max = max(1, 8192 * 4096 // C)
            if rng.random() < 0.5 and C <= 1024:
                H = _log_int(rng, 4, 224)
                W = H if rng.random() < 0.6 else max(4, int(round(H * rng.uniform(0.5, 2.0))))
                if H * W > rows_max:
                    continue
                B = _log_int(rng, 1, max(1, min(512, rows_max // (H * W))))
            else:
                B, H, W = _log_int(rng, 1, min(rows_max, 1 << 17)), 0, 0
            return dict(op=op, dtype=dtype, B=B, C=C, H=H, W=W, params=rng.choice(["f32", dtype]))
        if op == "orthogonalize":
            kind = rng.choice(["matrix", "conv", "batch"])
            if kind == "conv":
                K = rng.choice([1, 3, 3, 3, 5])
                shape = (_log_int(rng, 8, 512), _log_int(rng, 1, 512), K, K)
            else:
                shape = (_log_int(rng, 1, 4096), _log_int(rng, 1, 4096))
                if kind == "batch":
                    shape = (_log_int(rng, 2, 32),) + shape
            c = dict(op=op, dtype=dtype, shape=":".join(map(str, shape)))
        else:
            layers = []
            width = rng.choice([16, 24, 32, 48, 64, 96, 128])
            for _ in range(_log_int(rng, 1, 24)):
                K = rng.choice([1, 3, 3, 3, 5])
                growth = [width * g for g in (1, 1, 2, 4)]
                layers.append((rng.choice(growth), rng.choice(growth), K, K) if rng.random() < 0.8 else (_log_int(rng, 10, 2048), rng.choice(growth)))
            c = dict(op=op, dtype=dtype, layers=" ".join(":".join(map(str, s)) for s in layers))
        if work(c)["flops"] <= flops_max:
            return c


def _gradient(gen, shape):
    """A gradient: a few directions above noise, rows of different size, dense in the library's layout of its rank."""
    batch, rows, cols = _matrices(shape)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    few = min(8, rows, cols)
    g = rnd(batch, rows, cols).add_((2.0 * rnd(batch, rows, few)) @ rnd(batch, few, cols) / math.sqrt(few))
    g = g.mul_(rnd(batch, rows, 1).mul_(0.5).exp_()).mul_(1e-3)
    return _as_weights(g, shape)


def _as_weights(g, shape):
    """(batch, rows, columns) -> a tensor of `shape`: the columns of a convolution's rows lie as (KH, KW, Cin)."""
    if len(shape) <= 3:
        return g.reshape(shape)
    Cout, Cin, KH, KW = shape
    return g.reshape(Cout, KH, KW, Cin).permute(0, 3, 1, 2)


def _as_matrices(t):
    if t.dim() == 4:
        return t.permute(0, 2, 3, 1).reshape(1, t.shape[0], -1)
    return t.reshape(_matrices(tuple(t.shape)))


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = _DTYPES[c["dtype"]]
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    s = dict(op=c["op"])
    if c["op"] in ("norm", "norm_backward"):
        C, params = c["C"], _DTYPES[c["params"]]
        shape = (c["B"], c["H"], c["W"], C) if c["H"] else (c["B"], C)
        image = (lambda t: t.permute(0, 3, 1, 2)) if c["H"] else (lambda t: t)
        loud = 1.0 + 9.0 * (torch.rand(C, generator=gen, device="cuda") < 0.02).float()
        s["X"] = image((rnd(*shape).mul_(loud).add_(0.5 + 0.5 * rnd(C))).to(dtype))
        s["weight"], s["bias"] = (1.0 + 0.2 * rnd(C)).to(params), (0.1 * rnd(C)).to(params)
        if c["op"] == "norm_backward":
            s["dY"] = image(rnd(*shape).mul_(0.1).to(dtype))
            _, s["mean"], s["rstd"] = _norm_plain(s["X"], s["weight"], s["bias"])      # kept since the forward pass
    elif c["op"] == "orthogonalize":
        s["G"] = _gradient(gen, _shape(c["shape"])).to(dtype)
    else:
        s["W"], s["dW"], s["M"] = [], [], []
        for shape in _layers(c["layers"]):
            _, rows, cols = _matrices(shape)
            s["W"].append(_as_weights((2.0 / cols) ** 0.5 * rnd(1, rows, cols), shape).to(dtype))
            s["dW"].append(_gradient(gen, shape))                                      # the library's estimates are float whatever the weights' type
            s["M"].append(_gradient(gen, shape))
    return s


def _channels_last(t):
    return t.movedim(1, -1) if t.dim() > 2 else t


def _channels_second(t):
    return t.movedim(-1, 1) if t.dim() > 2 else t


def _norm_plain(X, weight, bias):
    x = _channels_last(X).float()
    mean = x.sum(-1, keepdim=True) / x.shape[-1]
    x = x - mean
    rstd = 1.0 / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + _NORM_EPS)
    y = x * rstd * weight.float() + bias.float()
    return _channels_second(y.to(X.dtype)), mean.squeeze(-1), rstd.squeeze(-1)


def _norm_backward_plain(dY, X, mean, rstd, weight):
    dy, x = _channels_last(dY).float(), _channels_last(X).float()
    rstd = rstd.unsqueeze(-1)
    xh = (x - mean.unsqueeze(-1)) * rstd
    g = dy * weight.float()
    C = x.shape[-1]
    dx = rstd * (g - g.sum(-1, keepdim=True) / C - xh * ((g * xh).sum(-1, keepdim=True) / C))
    rows = tuple(range(dy.dim() - 1))
    return _channels_second(dx.to(X.dtype)), (dy * xh).sum(rows), dy.sum(rows)


def _orthogonal(G):
    """Newton-Schulz steps on (batch, rows, columns), in the type of G."""
    tall = G.shape[1] > G.shape[2]
    X = G.transpose(1, 2) if tall else G
    X = X / torch.sqrt((X * X).sum((1, 2), keepdim=True)).clamp(min=_EPS)
    a, b, c = _COEFFICIENTS
    for _ in range(_STEPS):
        A = X @ X.transpose(1, 2)
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.transpose(1, 2) if tall else X


def _muon_plain(W, dW, M):
    M.mul_(_MOMENTUM).add_((1 - _MOMENTUM) * dW.float())
    O = _as_weights(_orthogonal(_as_matrices(_MOMENTUM * M + (1 - _MOMENTUM) * dW.float())), tuple(W.shape))
    _, rows, cols = _matrices(tuple(W.shape))
    W.copy_(W.float() * (1 - _LR * _DECAY) - (_LR * math.sqrt(max(1.0, rows / cols))) * O)


def run(state):
    s = state
    if own:
        from paper_2106_06998_b200 import binding as xb
        if s["op"] == "norm":
            Y, mean, rstd = xb.xconv_layernorm(s["X"], s["weight"], s["bias"], eps=_NORM_EPS)
            return {"Y": Y, "mean": mean, "rstd": rstd}
        if s["op"] == "norm_backward":
            dX, dweight, dbias = xb.xconv_layernorm_backward(s["dY"], s["X"], s["mean"], s["rstd"], s["weight"])
            return {"dX": dX, "dweight": dweight, "dbias": dbias}
        if s["op"] == "orthogonalize":
            return {"O": xb.xconv_orthogonalize(s["G"], steps=_STEPS, coefficients=_COEFFICIENTS, eps=_EPS)}
        xb.xconv_muon_step(s["W"], s["dW"], s["M"], lr=_LR, momentum=_MOMENTUM, weight_decay=_DECAY, steps=_STEPS, coefficients=_COEFFICIENTS, eps=_EPS)
        return {"W": s["W"], "M": s["M"]}
    if s["op"] == "norm":
        Y, mean, rstd = _norm_plain(s["X"], s["weight"], s["bias"])
        return {"Y": Y, "mean": mean, "rstd": rstd}
    if s["op"] == "norm_backward":
        dX, dweight, dbias = _norm_backward_plain(s["dY"], s["X"], s["mean"], s["rstd"], s["weight"])
        return {"dX": dX, "dweight": dweight, "dbias": dbias}
    if s["op"] == "orthogonalize":
        G = s["G"]
        return {"O": _as_weights(_orthogonal(_as_matrices(G).float()), tuple(G.shape)).to(G.dtype)}
    for W, dW, M in zip(s["W"], s["dW"], s["M"]):
        _muon_plain(W, dW, M)
    return {"W": s["W"], "M": s["M"]}


def _exact_polynomial(G):
    """The orthogonalised matrices by singular values: each step maps a singular value x to a x + b x^3 + c x^5."""
    U, sv, Vh = torch.linalg.svd(G, full_matrices=False)
    sv = sv / sv.square().sum(-1, keepdim=True).sqrt().clamp(min=_EPS)
    a, b, c = _COEFFICIENTS
    for _ in range(_STEPS):
        q = sv * sv
        sv = sv * (a + q * (b + q * c))
    return (U * sv.unsqueeze(-2)) @ Vh


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] in ("norm", "norm_backward"):
        axis = 1
        C = case["C"]
        shape = [1, C] + [1] * (s["X"].dim() - 2)
        x, w, b = s["X"].double(), s["weight"].double().view(shape), s["bias"].double().view(shape)
        if s["op"] == "norm":
            var, mean = torch.var_mean(x, dim=axis, correction=0, keepdim=True)
            rstd = (var + _NORM_EPS) ** -0.5
            return {"Y": (x - mean) * rstd * w + b, "mean": mean.squeeze(axis), "rstd": rstd.squeeze(axis)}
        dy = s["dY"].double()
        mean, rstd = s["mean"].double().unsqueeze(axis), s["rstd"].double().unsqueeze(axis)
        xh = (x - mean) * rstd
        others = [d for d in range(x.dim()) if d != axis]
        out = {"dweight": (dy * xh).sum(others), "dbias": dy.sum(others)}
        dy = dy * w
        out["dX"] = rstd * (dy - dy.mean(axis, keepdim=True) - xh * (dy * xh).mean(axis, keepdim=True))
        return out
    sizes = [_matrices(tuple(t.shape)) for t in ([s["G"]] if s["op"] == "orthogonalize" else s["W"])]
    if sum(n * min(r, c) ** 2 * max(r, c) for n, r, c in sizes) > 1.2e10:
        return None                                          # (singular values of so much take longer than they are worth)
    if s["op"] == "orthogonalize":
        return {"O": _as_weights(_exact_polynomial(_as_matrices(s["G"]).double()), tuple(s["G"].shape))}
    out = {"W": [], "M": []}
    for (_, rows, cols), W, dW, M in zip(sizes, s["W"], s["dW"], s["M"]):
        g = dW.double()
        m = M.double() + (1 - _MOMENTUM) * (g - M.double())
        O = _as_weights(_exact_polynomial(_as_matrices(g + _MOMENTUM * (m - g))), tuple(W.shape))
        out["M"].append(m)
        out["W"].append(W.double() - _LR * (_DECAY * W.double() + max(1.0, rows / cols) ** 0.5 * O))
    return out


def work(case):
    """Inputs read once, outputs written once; of the products the symmetric ones counted by their lower halves."""
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["op"] in ("norm", "norm_backward"):
        rows, C = c["B"] * max(1, c["H"] * c["W"]), c["C"]
        ps = 4 if c["params"] == "f32" else 2
        if c["op"] == "norm":
            return {"bytes": 2 * es * rows * C + 2 * ps * C + 8 * rows, "flops": 8 * rows * C}
        return {"bytes": 3 * es * rows * C + ps * C + 8 * rows + 8 * C, "flops": 14 * rows * C}
    nbytes, flops = 0, 0
    for shape in [_shape(c["shape"])] if c["op"] == "orthogonalize" else _layers(c["layers"]):
        batch, rows, cols = _matrices(shape)
        n, m = min(rows, cols), max(rows, cols)
        flops += batch * _STEPS * (3 * n * n * m + n * n * n)
        nbytes += batch * rows * cols * (2 * es if c["op"] == "orthogonalize" else 2 * es + 12)
    return {"bytes": nbytes, "flops": flops}
