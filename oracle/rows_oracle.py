"""Plain oracle of what rows of heads go through on their way (64-bit numpy, no code shared with the GPU path): norm and rotation by
position, and the 8-bit form of a cache's rows.  The rules are those of ``include/np.h``."""
import numpy as np


def rotate(x, gain, eps, pos, freq, neighbours):
    """x [heads][head_dim] float64 of one token; gain [head_dim] or None; freq [rot_dim / 2]."""
    x = np.asarray(x, np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    half = len(freq)
    if half == 0:
        return x
    t = float(pos) * np.asarray(freq, np.float64)
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if neighbours else (x[..., :half], x[..., half:2 * half])
    u, w = a * np.cos(t) - b * np.sin(t), b * np.cos(t) + a * np.sin(t)
    out = x.copy()
    if neighbours:
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = u, w
    else:
        out[..., :half], out[..., half:2 * half] = u, w
    return out


def e4m3_values():
    """What the 256 bytes stand for."""
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = np.nan if e == 15 and m == 7 else (m / 8.0 * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7))
        v[b] = -x if b & 128 else x
    return v


def hold(x):
    """Rows [..., head_dim] float64 -> (values as held, times their power of two; biased exponents [...])."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    top = np.where(fine, np.abs(x), 0.0).max(-1)
    e = np.full(top.shape, -60)
    for k in range(-60, 120):                       # the least exponent whose 448 * 2^e is not below the largest
        e = np.where(top > 448.0 * 2.0 ** k, k + 1, e)
    scale = 2.0 ** e.astype(np.float64)[..., None]
    y = np.where(fine, x, 0.0) / scale
    grid = np.sort(e4m3_values()[:127])             # 0 and the positive numbers, by rising byte
    a = np.abs(y)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up = (grid[hi] - a < a - grid[lo]) | ((grid[hi] - a == a - grid[lo]) & (hi % 2 == 0))
    r = np.where(up, grid[hi], grid[lo]) * np.sign(y)
    return np.where(fine, r * scale, np.nan), (e + 127).astype(np.int64)
