"""Operators at the end of one block and the beginning of the next: dropout whose mask is drawn from a seed and never stored, the residual's addition, the
root-mean-square norm over the channels, forward and backward, and its output in 8 bits with scales.

A case is one pass:

  rmsnorm            Y, rstd and, where something is added to X, the sum H
  rmsnorm_quantized  the same with Y in 8 bits, and the values that these stand for, as the layer that reads them takes them
  rmsnorm_backward   dX, dweight and, where X was dropped out, the residual's gradient
  dropout            Y, of single values or of whole channels, with or without a residual
  dropout_backward   dX

Tensors are on the GPU as the library takes them: images channels-last, tokens row-major.  Activations have a few channels that are ten times the others.

The mask: u, 32 bits, of value c of a row of mask row m (the row's number; that of its image where whole channels are dropped) is made of two halves of 16 bits, both the
(c mod 8)-th (of four words, the low one first) of the Philox-4x32-10 block with counter words (b, b >> 32, w, 0), b = m ceil(C / 8) + c div 8, and the seed as key;
w = 3 for the upper half and 4 for the lower one.  A value is dropped where u < floor(p 2^32), and divided by 1 - p elsewhere.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-6
_LARGEST = {"e4m3": 448.0, "int8": 127.0}
_LEAST = 2.0 ** -100                           # of a group's largest value, for its scale


def _case(name, op, dtype, B, C, H=0, W=0, params="f32", residual=True, p=0.0, channels=False, q="", group=0):
    """H = 0: a matrix of B tokens of C values; else a channels-last image batch.  params: the type of the weight.  residual: added to X (backward: the sum's own
    gradient comes in).  p, channels: dropout of values or of whole channels.  q, group: 8 bits, and the values that share a scale (0: the row)."""
    return dict(name=name, op=op, dtype=dtype, B=B, C=C, H=H, W=W, params=params, residual=residual, p=p, channels=channels, q=q, group=group)


def listed():
    return [
        # A single token of a decoder: latency.
        _case("rms_token_bf16", "rmsnorm", "bf16", 1, 4096, params="bf16"),
        # Many tokens of a wide model: the largest norm.
        _case("rms_tokens_bf16", "rmsnorm", "bf16", 8192, 4096, params="bf16"),
        # The last, short batch of an epoch on images of odd size with an odd number of channels, trained with dropout: no row is aligned.
        _case("rms_ragged_dropout_f16", "rmsnorm", "f16", 50, 97, 35, 27, params="f16", p=0.1),
        # A batch of single tokens on its way into products of 8-bit values, one scale a token.
        _case("quantized_batch_e4m3", "rmsnorm_quantized", "bf16", 32, 4096, params="bf16", q="e4m3"),
        # Tokens of a prompt, a scale for every 128 values.
        _case("quantized_tokens_e4m3", "rmsnorm_quantized", "bf16", 8192, 2048, params="bf16", q="e4m3", group=128),
        # Activations of a residual network's first stage, in float, kept in 8 bits between the passes.
        _case("quantized_image_int8", "rmsnorm_quantized", "f32", 128, 64, 32, 32, q="int8"),
        # A small image batch, backward.
        _case("rms_small_backward_f32", "rmsnorm_backward", "f32", 8, 96, 14, 14, residual=False),
        # Many tokens of a wide model, backward, with the gradient that comes in past the norm.
        _case("rms_tokens_backward_bf16", "rmsnorm_backward", "bf16", 8192, 4096, params="bf16"),
        # Images of odd size and an odd number of channels, backward, through the dropout.
        _case("rms_ragged_backward_f16", "rmsnorm_backward", "f16", 50, 97, 35, 27, params="f16", p=0.1),
        # The end of a residual block on a large batch of wide images: the largest case.
        _case("dropout_image_bf16", "dropout", "bf16", 512, 256, 28, 28, p=0.1),
        # Whole channels of images of odd size, in front of a convolution.
        _case("dropout_channels_f16", "dropout", "f16", 50, 97, 35, 27, residual=False, p=0.2, channels=True),
        # A small image batch, backward: latency.
        _case("dropout_small_backward_f32", "dropout_backward", "f32", 8, 96, 14, 14, residual=False, p=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more pass of the same ranges: 8 to 8192 channels, on and off the multiples of 8, one row up to the bytes of the largest listed case."""
    bytes_max = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["rmsnorm", "rmsnorm", "rmsnorm_quantized", "rmsnorm_quantized", "rmsnorm_backward", "rmsnorm_backward", "dropout", "dropout_backward"])
        dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
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
        residual = rng.random() < 0.7
        p = rng.choice([0.1, 0.2, 0.5, rng.uniform(0.01, 0.9)])
        if op.startswith("rmsnorm") and rng.random() < 0.6:
            p = 0.0
        c = _case("", op, dtype, B, C, H, W, rng.choice(["f32", dtype]), residual and op != "dropout_backward", p, bool(p and H and rng.random() < 0.3))
        if op == "rmsnorm_quantized":
            c["q"], c["group"] = rng.choice(["e4m3", "int8"]), rng.choice([0, 0, 32, 64, 128])
        del c["name"]
        if work(c)["bytes"] <= bytes_max:
            return c


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, C = _DTYPES[c["dtype"]], c["C"]
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    shape = (c["B"], c["H"], c["W"], C) if c["H"] else (c["B"], C)
    image = (lambda t: t.permute(0, 3, 1, 2)) if c["H"] else (lambda t: t)
    loud = 1.0 + 9.0 * (torch.rand(C, generator=gen, device="cuda") < 0.02).float()
    s = dict(case=c, seed=(seed * 0x9E3779B97F4A7C15 + 12345) % 2 ** 64)
    s["weight"] = (1.0 + 0.2 * rnd(C)).to(_DTYPES[c["params"]])
    s["X"] = image(rnd(*shape).mul_(loud).to(dtype))
    if c["residual"]:
        s["R"] = image(rnd(*shape).mul_(2.0 * loud).to(dtype))
    if c["op"] == "rmsnorm_backward":
        s["dY"] = image(rnd(*shape).mul_(0.1).to(dtype))
        s["H"], s["rstd"] = s.pop("X"), None
        if c["residual"]:
            s["dH"] = s.pop("R").mul_(0.05)
        s["rstd"] = _norm_plain(s["H"].float(), s["weight"])[1]         # kept since the forward pass
    elif c["op"] == "dropout_backward":
        s["dY"] = s.pop("X").mul_(0.1)
    return s


def _last(t):
    return t.movedim(1, -1) if t.dim() > 2 else t


def _second(t):
    return t.movedim(-1, 1) if t.dim() > 2 else t


def _philox_plain(blocks, word, seed):
    """The eight halves of 16 bits of the blocks, (..., 8)."""
    c0, c1, c2, c3 = blocks & 0xFFFFFFFF, blocks >> 32, torch.full_like(blocks, word), torch.zeros_like(blocks)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                         # (64 bits that wrap around: the upper ones come with a sign)
        c0, c1, c2, c3 = ((b >> 32) & 0xFFFFFFFF) ^ c1 ^ k0, b & 0xFFFFFFFF, ((a >> 32) & 0xFFFFFFFF) ^ c3 ^ k1, a & 0xFFFFFFFF
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).flatten(-2)


def _kept_plain(c, seed, device):
    """The mask of a case, channels last: true where a value is kept."""
    C, groups = c["C"], (c["C"] + 7) // 8
    masks = c["B"] if c["channels"] else c["B"] * max(1, c["H"] * c["W"])
    blocks = torch.arange(masks * groups, device=device).view(masks, groups)
    u = (_philox_plain(blocks, 3, seed) << 16) + _philox_plain(blocks, 4, seed)
    kept = u.view(masks, groups * 8)[:, :C] >= math.floor(c["p"] * 2.0 ** 32)
    if not c["H"]:
        return kept
    return kept.view(c["B"], 1, 1, C) if c["channels"] else kept.view(c["B"], c["H"], c["W"], C)


def _dropped_plain(t, c, seed):
    """t in floats, channels last, dropped out."""
    if not c["p"]:
        return t
    return torch.where(_kept_plain(c, seed, t.device), t / (1.0 - c["p"]), torch.zeros((), device=t.device, dtype=t.dtype))


def _sum_plain(s):
    h = _dropped_plain(_last(s["X"]).float(), s["case"], s["seed"])
    return h + _last(s["R"]).float() if s["case"]["residual"] else h


def _norm_plain(h, weight):
    """(y, rstd) of h in floats, channels second."""
    h = _last(h)
    rstd = 1.0 / torch.sqrt((h * h).sum(-1) / h.shape[-1] + _EPS)
    return h * rstd.unsqueeze(-1) * weight.to(h.dtype), rstd


def _groups(t, group):
    """(..., C) -> (..., groups, values), with zeros behind a row's last values."""
    C = t.shape[-1]
    group = group or C
    return torch.nn.functional.pad(t, (0, -C % group)).unflatten(-1, (-1, group))


def _quantized_plain(y, c):
    """(values, scales) of y, channels last, in 64 bits: a value next to the border of two 8-bit ones has to come out on its side."""
    M = _LARGEST[c["q"]]
    y = _groups(y, c["group"])
    scales = (y.abs().amax(-1).clamp(min=_LEAST) / M).float()
    q = y / scales.double().unsqueeze(-1)
    q = q.clamp(-M, M).float().to(torch.float8_e4m3fn).double() if c["q"] == "e4m3" else q.round().clamp(-M, M)
    return (q * scales.double().unsqueeze(-1)).flatten(-2)[..., :c["C"]], scales


def _values_type(dtype):
    return torch.bfloat16 if dtype == torch.float32 else dtype


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if own:
        from paper_2106_06998_b200 import binding as xb
        drop = dict(p=c["p"], seed=s["seed"], channels=c["channels"]) if c["p"] else {}
        if op == "rmsnorm":
            Y, H, rstd = xb.xconv_rmsnorm(s["X"], s["weight"], residual=s.get("R"), eps=_EPS, **drop)
            return {"Y": Y, "rstd": rstd, "H": H} if c["residual"] or drop else {"Y": Y, "rstd": rstd}
        if op == "rmsnorm_quantized":
            qdtype = torch.float8_e4m3fn if c["q"] == "e4m3" else torch.int8
            Q, scales, H, rstd = xb.xconv_rmsnorm_quantized(s["X"], s["weight"], residual=s.get("R"), eps=_EPS, qdtype=qdtype, group=c["group"], **drop)
            out = {"values": xb.xconv_dequantize(Q, scales, group=c["group"], dtype=_values_type(s["X"].dtype)), "scales": scales, "rstd": rstd}
            return {**out, "H": H} if c["residual"] or drop else out
        if op == "rmsnorm_backward":
            dX, dresidual, dweight = xb.xconv_rmsnorm_backward(s["dY"], s["H"], s["rstd"], s["weight"], dH=s.get("dH"), **drop)
            return {"dX": dX, "dresidual": dresidual, "dweight": dweight} if drop else {"dX": dX, "dweight": dweight}
        if op == "dropout":
            return {"Y": xb.xconv_dropout(s["X"], residual=s.get("R"), **drop)}
        return {"dX": xb.xconv_dropout_backward(s["dY"], **drop)}
    if op == "rmsnorm":
        h = _sum_plain(s)
        dtype = s["X"].dtype
        y, rstd = _norm_plain(_second(h), s["weight"])
        out = {"Y": _second(y.to(dtype)), "rstd": rstd}
        return {**out, "H": _second(h.to(dtype))} if c["residual"] or c["p"] else out
    if op == "rmsnorm_quantized":
        h = _sum_plain(s)
        dtype = s["X"].dtype
        y, rstd = _norm_plain(_second(h).double(), s["weight"])
        values, scales = _quantized_plain(y, c)
        out = {"values": _second(values.to(_values_type(dtype))), "scales": _second(scales), "rstd": rstd.float()}
        return {**out, "H": _second(h.to(dtype))} if c["residual"] or c["p"] else out
    if op == "dropout":
        return {"Y": _second(_sum_plain(s).to(s["X"].dtype))}
    dtype = s["dY"].dtype
    dy = _last(s["dY"]).float()
    if op == "dropout_backward":
        return {"dX": _second(_dropped_plain(dy, c, s["seed"]).to(dtype))}
    xh = _last(s["H"]).float() * s["rstd"].unsqueeze(-1)
    g = dy * s["weight"].float()
    dr = s["rstd"].unsqueeze(-1) * (g - xh * ((g * xh).sum(-1, keepdim=True) / c["C"]))
    if c["residual"]:
        dr = dr + _last(s["dH"]).float()
    out = {"dX": _second(_dropped_plain(dr, c, s["seed"]).to(dtype)), "dweight": (dy * xh).sum(tuple(range(dy.dim() - 1)))}
    return {**out, "dresidual": _second(dr.to(dtype))} if c["p"] else out


def _philox_exact(blocks, word, seed):
    """The blocks' words as halves, in numpy's unsigned numbers."""
    M = np.uint64(0xFFFFFFFF)
    x = [blocks & M, blocks >> np.uint64(32), np.full_like(blocks, word), np.zeros_like(blocks)]
    key = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
    for i in range(10):
        p0, p1 = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(p1 >> np.uint64(32)) ^ x[1] ^ key[0], p1 & M, (p0 >> np.uint64(32)) ^ x[3] ^ key[1], p0 & M]
        key = [(key[0] + np.uint64(0x9E3779B9)) & M, (key[1] + np.uint64(0xBB67AE85)) & M]
    return np.stack(x, -1).astype("<u4").view("<u2")


def _factor_exact(c, seed):
    """What the dropout multiplies by, in 64 bits, (B, 1 or pixels, C)."""
    pixels = 1 if c["channels"] else max(1, c["H"] * c["W"])
    words = (c["C"] + 7) // 8
    n, least = c["B"] * pixels * words, np.uint64(int(c["p"] * 2 ** 32))
    dropped = np.empty(n * 8, dtype=bool)
    for first in range(0, n, 1 << 15):
        blocks = np.arange(first, min(n, first + (1 << 15)), dtype=np.uint64)
        upper, lower = (_philox_exact(blocks, word, seed).astype(np.uint64).reshape(-1) for word in (3, 4))
        dropped[8 * first:8 * first + upper.size] = upper * np.uint64(65536) + lower < least
    return torch.from_numpy(~dropped).cuda().view(c["B"], pixels, words * 8)[:, :, :c["C"]].double().div_(1 - c["p"])


_E4M3 = torch.tensor([(8 + i % 8) * 2.0 ** (i // 8 - 10) if i >= 8 else i * 2.0 ** -9 for i in range(127)], dtype=torch.float64)


def _to_e4m3_exact(v):
    """The nearest 8-bit value of |v| <= 448 (1 + a little): of two at the same distance the one whose code is even."""
    table = _E4M3.to(v.device)
    a = v.abs().clamp(max=448.0)
    above = torch.bucketize(a, table).clamp(max=126)
    below = (above - 1).clamp(min=0)
    up, down = table[above] - a, a - table[below]
    code = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
    return torch.copysign(table[code], v)


def exact(case, seed):
    s, c = prepare(case, seed), case
    op, C, image = c["op"], c["C"], bool(c["H"])
    pixels = max(1, c["H"] * c["W"])
    flat = lambda t: (t.permute(0, 2, 3, 1) if image else t).reshape(c["B"], pixels, C).double()
    back = lambda t: t.reshape(c["B"], c["H"], c["W"], -1).permute(0, 3, 1, 2) if image else t.reshape(c["B"], -1)
    per_row = lambda t: t.reshape((c["B"], c["H"], c["W"]) if image else (c["B"],))
    factor = _factor_exact(c, s["seed"]) if c["p"] else 1.0
    w = s["weight"].double()
    if op == "dropout_backward":
        return {"dX": back(flat(s["dY"]) * factor)}
    if op == "rmsnorm_backward":
        dy, h, r = flat(s["dY"]), flat(s["H"]), s["rstd"].double().view(c["B"], pixels, 1)
        out = {"dweight": torch.einsum("bpc,bpc,bp->c", dy, h, r[..., 0])}
        dot = torch.einsum("bpc,bpc,c->bp", dy, h, w)[..., None] * r
        grad = r * dy * w - (r * r / C) * dot * h
        if c["residual"]:
            grad = grad + flat(s["dH"])
        out["dX"] = back(grad * factor)
        return {**out, "dresidual": back(grad)} if c["p"] else out
    h = flat(s["X"]) * factor
    if c["residual"]:
        h = h + flat(s["R"])
    if op == "dropout":
        return {"Y": back(h)}
    rstd = (h.square().mean(-1, keepdim=True) + _EPS) ** -0.5
    y = h * (rstd * w)
    out = {"rstd": per_row(rstd)}
    if c["residual"] or c["p"]:
        out["H"] = back(h)
    if op == "rmsnorm":
        return {**out, "Y": back(y)}
    M, group = _LARGEST[c["q"]], c["group"] or C
    parts = torch.split(y, group, -1)
    scale = torch.cat([t.abs().amax(-1, keepdim=True) for t in parts], -1).clamp(min=_LEAST) / M
    wide = scale.repeat_interleave(group, -1)[..., :C]
    q = y / wide
    q = _to_e4m3_exact(q) if c["q"] == "e4m3" else torch.round(q)
    return {**out, "values": back(q * wide), "scales": back(scale)}


def work(case):
    """Inputs read once, outputs written once; 8-bit values are both."""
    c = case
    es, ps = 4 if c["dtype"] == "f32" else 2, 4 if c["params"] == "f32" else 2
    rows, C, op = c["B"] * max(1, c["H"] * c["W"]), c["C"], c["op"]
    n = rows * C
    draws = 15 * n if c["p"] and not c["channels"] else 0                # operations on whole numbers: ten rounds of twelve for eight values
    if op in ("dropout", "dropout_backward"):
        return {"bytes": es * n * (3 if c["residual"] else 2), "flops": 2 * n + draws}
    if op == "rmsnorm_backward":
        tensors = 3 + bool(c["residual"]) + bool(c["p"])
        return {"bytes": es * n * tensors + ps * C + 4 * rows + 4 * C, "flops": 10 * n + draws}
    tensors = 1 + bool(c["residual"]) + bool(c["residual"] or c["p"])
    nbytes, flops = es * n * tensors + ps * C + 4 * rows, 5 * n + draws
    if op == "rmsnorm":
        return {"bytes": nbytes + es * n, "flops": flops}
    scales = rows * -(-C // (c["group"] or C))
    return {"bytes": nbytes + 2 * n + 8 * scales + 2 * n, "flops": flops + 4 * n}
