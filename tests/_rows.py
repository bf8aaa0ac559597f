"""The operators between the blocks in 64 bits, for their tests: the mask in numpy's unsigned numbers, the rest from the formulas."""
import numpy as np
import torch

HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}    # half a step, relative to the value
# Sums in float: a thread adds at most 64 values one after another and the threads' sums in ten steps, what goes in has a few roundings, the root and the products some more --
# at most 2^6 roundings of 2^-24 of the sum of the magnitudes in all.
SUMS = 2.0 ** -18
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}   # half a step below the normal values


def philox(blocks, word, seed):
    M = np.uint64(0xFFFFFFFF)
    x = [blocks & M, blocks >> np.uint64(32), np.full_like(blocks, word), np.zeros_like(blocks)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), b & M, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k1), a & M]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(x, -1)


def kept(rows, C, p, seed, per=1, first=0):
    """The mask of rows `first` on, (rows, C): true where a value is kept."""
    octets = (C + 7) // 8
    m = np.arange(first, first + rows, dtype=np.uint64) // np.uint64(per)
    blocks = (m[:, None] * np.uint64(octets) + np.arange(octets, dtype=np.uint64)[None]).reshape(-1)
    words = [philox(blocks, w, seed % 2 ** 64) for w in (3, 4)]
    halves = [np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(rows, octets * 8)[:, :C] for w in words]
    u = (halves[0] << np.uint64(16)) + halves[1]
    return torch.from_numpy(u >= np.uint64(int(p * 2.0 ** 32)))


def last(t):
    """(rows, C) of a tensor of the library's layout, in 64 bits on the host."""
    t = t.detach().movedim(1, -1) if t.dim() >= 4 else t.detach()
    return t.reshape(-1, t.shape[-1]).cpu().double()


def per_of(X, channels):
    if not channels:
        return 1
    shape = list(X.shape)
    shape.pop(1 if X.dim() >= 4 else -1)
    return max(1, int(np.prod(shape[1:])))


def dropped(x, p, seed, per=1):
    """drop(x) of rows in 64 bits."""
    if p == 0:
        return x
    scale = 0.0 if p == 1 else 1.0 / (1.0 - p)
    return torch.where(kept(x.shape[0], x.shape[1], p, seed, per), x * scale, torch.zeros((), dtype=torch.float64))


def close(name, got, want, tol):
    """Every value within its own tolerance; what is not finite in the same places."""
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), f"{name}: not finite in other places"
    off = torch.where(fine, (got - want).abs() - tol, torch.full_like(want, -1.0))
    worst = int(off.argmax()) if off.numel() else 0
    assert off.numel() == 0 or float(off.max()) <= 0, f"{name}: value {worst} is {got.flatten()[worst]}, not {want.flatten()[worst]} within {tol.flatten()[worst]}"


def norm(X, weight, residual, eps, p=0.0, seed=0, channels=False):
    """(y, h, rstd) in 64 bits, and how far those of float arithmetic may be off before they are rounded to their types."""
    x = dropped(last(X), p, seed, per_of(X, channels))
    r = last(residual) if residual is not None else torch.zeros_like(x)
    w = weight.detach().cpu().double() if weight is not None else torch.ones(x.shape[1], dtype=torch.float64)
    h = x + r
    rstd = (h.square().mean(1) + eps) ** -0.5
    y = h * rstd[:, None] * w
    h_off = 2.0 ** -22 * (x.abs() + r.abs())
    # (the sum of squares moves with h: relative to its root by at most |h_off| / |h| in the 2-norm)
    moved = h_off.square().sum(1).sqrt() * rstd / x.shape[1] ** 0.5
    return (y, h, rstd), ((h_off * rstd[:, None] * w.abs() + (SUMS + moved[:, None]) * y.abs()), h_off, (SUMS + moved) * rstd)


def norm_backward(dY, H, rstd, weight, dH, p=0.0, seed=0, channels=False):
    """(dx, dr, dweight) in 64 bits, and how far those of float arithmetic may be off before they are rounded."""
    dy, h, r = last(dY), last(H), rstd.detach().cpu().double().reshape(-1, 1)
    w = weight.detach().cpu().double() if weight is not None else torch.ones(h.shape[1], dtype=torch.float64)
    d = last(dH) if dH is not None else torch.zeros_like(h)
    xh, g = h * r, dy * w
    dr = d + r * (g - xh * (g * xh).mean(1, keepdim=True))
    off = SUMS * (d.abs() + r * (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True)))
    dx = dropped(dr, p, seed, per_of(H, channels))
    scale = 1.0 if p in (0, 1) else 1 / (1 - p)
    return (dx, dr, (dy * xh).sum(0)), (off * scale, off, 2.0 ** -17 * (dy * xh).abs().sum(0))


def rounded(want, off, dtype):
    """The tolerance of values that are rounded to `dtype` once, after an error of `off`."""
    return off * (1 + HALF[dtype]) + HALF[dtype] * want.abs() + TINY[dtype]
