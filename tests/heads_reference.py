"""Head norms, rotation and pages of 4-bit numbers from their definitions, in 64 bits on the CPU; and the bound that rows are held to.

Rows: a number is computed in 64 bits and rounded to fp32, then to the rows' type.  Against the formula it is off by at most half a step of the type, eps / 2 of
itself, and half a step of fp32 before that, 2^-24; the 64-bit sums add less than 2^-44 of the two numbers that are turned (128 squares summed in any order, a root,
a quotient and two products, each 2^-53).
"""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def turned(x, heads, weight, eps, positions, rotation, pairs):
    """(values, bound) [T, heads * D] in 64 bits; rows of negative position are NaN (they are not written)."""
    T, D = x.shape[0], x.shape[1] // heads
    h = x.double().reshape(T, heads, D)
    if weight is not None:
        h = h / torch.sqrt((h * h).mean(-1, keepdim=True) + float(np.float32(eps))) * weight.double()
    size = h.abs()
    if rotation is not None:
        R = rotation.shape[1]
        at = positions.long().clamp(0, rotation.shape[0] - 1)
        c, s = rotation.double()[at][:, None, :R // 2], rotation.double()[at][:, None, R // 2:]
        p = torch.arange(R // 2)
        i, j = (p, p + R // 2) if pairs == 0 else (2 * p, 2 * p + 1)
        out, most = h.clone(), h.abs()
        out[..., i], out[..., j] = h[..., i] * c - h[..., j] * s, h[..., j] * c + h[..., i] * s
        most[..., i] = most[..., j] = h[..., i].abs() + h[..., j].abs()
        h, size = out, most
    half = torch.finfo(x.dtype).eps / 2
    bound = (half + 2.0 ** -24) * h.abs() * 1.001 + 2.0 ** -44 * size + 1e-40
    h, bound = h.reshape(T, -1), bound.reshape(T, -1)
    if positions is not None:
        h[positions < 0] = float("nan")
    return h, bound


def check_rows(got, before, want, bound, real):
    """Rows of `real` within their bounds, the others as before; infinities and NaN where they belong."""
    got, before = got.cpu(), before.cpu()
    assert torch.equal(got[~real].view(torch.uint8), before[~real].view(torch.uint8)), "a row of padding was written"
    g, w, b = got[real].double(), want[real], bound[real]
    fine = torch.isfinite(w)
    assert torch.equal(torch.isnan(g), torch.isnan(w)) and torch.equal(g[~fine & ~torch.isnan(w)], w[~fine & ~torch.isnan(w)])
    over = ((g - w).abs() / b)[fine]
    assert over.numel() == 0 or over.max() <= 1.0, f"{over.max():.4f} times the bound"


def to_four(x):
    """x [..., D] (numbers of the rows' type, as float64): numbers' codes [..., D] and powers' bytes [..., D / 32], by search."""
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(b).all(-1)
    e = np.full(top.shape, 125)
    for k in range(124, -126, -1):                            # the least power at which the largest is below 7
        e = np.where(top < 7 * 2.0 ** k, k, e)
    y = np.abs(np.where(bad[..., None], 0, b)) / (2.0 ** e.astype(np.float64))[..., None]
    d = np.abs(y[..., None] - GRID)
    near = d == d.min(-1, keepdims=True)                      # one, or the two that y is between
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(near.sum(-1) == 2, even.argmax(-1), near.argmax(-1)) + 8 * np.signbit(b)
    return np.where(bad[..., None], 0, code).reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def from_four(codes, powers):
    sign = np.where(codes >= 8, -1.0, 1.0)
    scale = np.where(powers == 255, np.nan, 2.0 ** (powers.astype(np.float64) - 127))
    return (sign * GRID[codes & 7]).reshape(*codes.shape[:-1], -1, 32).__mul__(scale[..., None]).reshape(codes.shape)


def split(cache, dim):
    """Cache bytes [pages, heads, page, dim / 2 + dim / 32] (NumPy): codes [pages, heads, page, dim] and powers [pages, heads, page, dim / 32]."""
    n, h, page, _ = cache.shape
    flat = cache.reshape(n, h, -1)
    b = flat[..., :page * dim // 2].reshape(n, h, page, dim // 2)
    return np.stack([b & 15, b >> 4], -1).reshape(n, h, page, dim), flat[..., page * dim // 2:].reshape(n, h, page, dim // 32)


def join(codes, powers):
    n, h, page, dim = codes.shape
    b = (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)
    return np.concatenate([b.reshape(n, h, -1), powers.reshape(n, h, -1).astype(np.uint8)], -1).reshape(n, h, page, dim // 2 + dim // 32)


def values(cache, dim):
    """Values [pages, heads, page, dim] of a cache's bytes, in 64 bits."""
    return from_four(*split(cache, dim))
