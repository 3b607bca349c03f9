"""Definitions in 64 bits, on the CPU, of head norms with rotary positions, of 4-bit records and of attention over them."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def norm_rope(x, positions, inv_freq, weight=None, offset=0.0, eps=1e-6, norm=True, axes_of=None, interleaved=False, mscale=1.0):
    """x [T, heads, d] -> (result, size): the result in 64 bits and, for error bounds, |x| + |y| of an element's pair."""
    x = x.double().cpu().numpy()
    T, _, d = x.shape
    if norm:
        with np.errstate(all="ignore"):
            x = x / np.sqrt((x * x).sum(-1, keepdims=True) / d + eps)
        if weight is not None:
            x = x * (offset + weight.double().cpu().numpy())
    f = inv_freq.double().cpu().numpy()
    r = 2 * len(f)
    pos = positions.cpu().numpy().reshape(-1, T).astype(np.float64)
    axes_of = np.zeros(len(f), int) if axes_of is None else axes_of.cpu().numpy()
    angle = (pos[axes_of].T * f)[:, None]
    c, s = np.cos(angle), np.sin(angle)
    out, size = x.copy(), np.abs(x)
    ix, iy = (np.arange(0, r, 2), np.arange(1, r, 2)) if interleaved else (np.arange(r // 2), np.arange(r // 2, r))
    a, b = x[..., ix], x[..., iy]
    out[..., ix], out[..., iy] = mscale * (a * c - b * s), mscale * (a * s + b * c)
    size[..., ix] = size[..., iy] = abs(mscale) * (np.abs(a) + np.abs(b))
    return out, size


def quantised(x):
    """x [.., d] (64-bit numpy) -> codes [.., d], scale bytes [.., d / 32]."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(b).max(-1)                                       # (NaN wins)
    finite = np.isfinite(top)
    e = np.frexp(np.where(finite & (top > 0), top, 1.0))[1] - 1   # floor(log2)
    scale = np.where(finite & (top > 0), np.maximum(e - 2, -127), -127) + 127
    y = np.abs(np.where(finite[..., None], b, 0.0)) / np.ldexp(1.0, scale - 127)[..., None]
    code = np.zeros(y.shape, int)
    for i in range(7):
        middle = (GRID[i] + GRID[i + 1]) / 2
        code = np.where((y > middle) | ((y == middle) & (i % 2 == 1)), i + 1, code)   # odd codes have an odd mantissa
    code = code + 8 * np.signbit(np.where(finite[..., None], b, 0.0))
    return code.reshape(x.shape), np.where(finite, scale, 255)


def values(codes, scales):
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales - 127))
    return v * np.repeat(s, 32, -1)


def unpacked(cache, page, d):
    """uint8 [pages, Hkv, record] -> (codes [pages, Hkv, P, d], scales [pages, Hkv, P, d / 32]) of K and of V."""
    c = cache.cpu().numpy().astype(int)
    n, h, _ = c.shape
    half, few = page * d // 2, page * d // 32
    k = c[..., :half].reshape(n, h, page, d // 2)
    v = c[..., half:2 * half].reshape(n, h, page // 8, 16, 8, d // 32).swapaxes(3, 4).reshape(n, h, page, d // 2)
    res = []
    for i, x in enumerate((k, v)):
        codes = np.stack([x & 15, x >> 4], -1).reshape(n, h, page, d)
        at = 2 * half + i * few
        res.append((codes, c[..., at:at + few].reshape(n, h, d // 32, page).swapaxes(2, 3)))
    return res


def attention(q, k, v, n_ctx, scale):
    """q [n, Hq, d], k and v [len, Hkv, d] (64-bit numpy); row i sees keys j <= n_ctx + i.  (out, lse, sum p |v|, largest sum |q k| scale)"""
    n, hq, d = q.shape
    G = hq // k.shape[1]
    out, mass = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, size = np.full((n, hq), -np.inf), np.zeros((n, hq))
    for h in range(hq):
        kk, vv = k[:, h // G], v[:, h // G]
        for i in range(n):
            seen = n_ctx + i + 1
            if seen <= 0:
                continue
            x = kk[:seen] @ q[i, h] * scale
            top = x.max()
            p = np.exp(x - top)
            lse[i, h] = top + np.log(p.sum())
            p /= p.sum()
            out[i, h], mass[i, h] = p @ vv[:seen], p @ np.abs(vv[:seen])
            size[i, h] = (np.abs(kk[:seen]) @ np.abs(q[i, h])).max() * abs(scale)
    return out, lse, mass, size
