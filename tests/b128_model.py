"""Plain numpy / float64 model of the 8-bit form with a Float32 scale for each block of 128, and of the RMS norm, from their definitions."""
import numpy as np

FMAX = {0: np.float32(448.0), 1: np.float32(57344.0)}
E4M3, E5M2 = 0, 1


def table(fmt):
    """The values of codes 0 .. 255."""
    bits, bias = (3, 7) if fmt == E4M3 else (2, 15)
    c = np.arange(256)
    field, low = (c & 127) >> bits, c & ((1 << bits) - 1)
    v = np.where(field == 0, low * 2.0 ** (1 - bias - bits), (1 + low / (1 << bits)) * 2.0 ** (field - float(bias)))
    if fmt == E4M3:
        v[(c & 127) == 127] = np.nan
    else:
        v[(c & 127) == 124] = np.inf
        v[(c & 127) > 124] = np.nan
    return np.where(c >= 128, -v, v)


def nearest(p, fmt):
    """Codes of the elements nearest to the Float32 products p (ties to even), clamped; NaN and infinity as the format has them."""
    last = 126 if fmt == E4M3 else 123
    v = table(fmt)[:last + 1]
    a = np.abs(p.astype(np.float64))
    fin = np.where(np.isfinite(a), a, 0.0)
    up = np.clip(np.searchsorted(v, fin), 1, last)                # v[up - 1] < fin <= v[up], as far as there is one
    lo, hi = fin - v[up - 1], v[up] - fin
    code = np.where((hi < lo) | ((hi == lo) & (up % 2 == 0)), up, up - 1)
    code = np.where(fin >= v[last], last, code)
    code = np.where(np.isnan(a), 127 if fmt == E4M3 else 126, np.where(np.isinf(a), 127 if fmt == E4M3 else 124, code))
    return (code | np.where(np.signbit(p), 128, 0)).astype(np.uint8)


def factor(amax, fmt):
    with np.errstate(divide="ignore", over="ignore"):
        q = np.minimum(FMAX[fmt] / amax.astype(np.float32), np.float32(2.0 ** 126))
    return (q.view(np.uint32) & np.uint32(0xFFFFFF00)).view(np.float32)


def blocks_of(x, tile):
    """x [R, L] filled up with zeros, as [R or R / 128, 1 or 128, blocks, 128]."""
    r, c = x.shape
    high = 128 if tile else 1
    full = np.zeros((-(-r // high) * high, -(-c // 128) * 128), dtype=np.float32)
    full[:r, :c] = x
    return full.reshape(full.shape[0] // high, high, -1, 128)


def quantize(x, axis, fmt, tile):
    """x: float32 [rows, cols].  Returns (codes, scales) as the library lays them out."""
    x = np.ascontiguousarray(x if axis == 1 else x.T)
    b = blocks_of(x, tile)
    mag = np.abs(b)
    amax = np.where(np.isfinite(mag), mag, 0).max((1, 3))
    f = factor(amax, fmt)
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        p = b * f[:, None, :, None]
    return nearest(p, fmt).reshape(-1, b.shape[2] * 128)[:x.shape[0]], np.float32(1) / f


def same_codes(a, b, fmt):
    """Equal, any NaN code equal to any other."""
    first = 127 if fmt == E4M3 else 125
    na, nb = (a & 127) >= first, (b & 127) >= first
    return bool(np.array_equal(na, nb) and np.array_equal(a[~na], b[~nb]))


def values(codes, scales, fmt, tile, dtype=np.float64):
    """elems * scales, [lines, length]."""
    s = np.repeat(scales, 128, 0)[:codes.shape[0]] if tile else scales
    v = table(fmt)[codes].astype(dtype).reshape(codes.shape[0], -1, 128)
    with np.errstate(invalid="ignore", over="ignore"):
        return (v * s.astype(dtype)[:, :, None]).reshape(codes.shape)


def norm_backward(dy, h, w, rstd, dh):
    dy, h, rstd = dy.astype(np.float64), h.astype(np.float64), rstd.astype(np.float64)[:, None]
    g = dy * (1.0 if w is None else w.astype(np.float64))
    xhat = h * rstd
    dx = rstd * (g - xhat * (g * xhat).mean(1, keepdims=True))
    return dx + (0 if dh is None else dh.astype(np.float64)), (dy * xhat).sum(0)
