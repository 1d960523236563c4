"""The operators of a feed-forward block in 8-bit floating point in IEEE double, each its definition written out: root-mean-square norm
with the residual's addition and its gradients, e4m3 codes with a power of two for each block of 128, products of such codes, and
the gated pair of projections with its gradients.  Inputs are what a caller stores; results are not rounded."""

import numpy as np

from .operators import activation, activation_slope


def _grid():
    """The magnitudes of codes 0 ... 126, from the format: 4 bits of exponent (bias 7), 3 of fraction."""
    values = []
    for code in range(127):
        e, m = code >> 3, code & 7
        values.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(values)


GRID = _grid()


def _blocks(x, squares):
    """x [rows, cols] -> zero-padded [row blocks, deep, pieces, 128]"""
    rows, cols = x.shape
    deep = 128 if squares else 1
    down, pieces = -(-rows // deep), -(-cols // 128)
    v = np.zeros((down * deep, pieces * 128))
    v[:rows, :cols] = x
    return v.reshape(down, deep, pieces, 128)


def fp8_quantize(x, squares=False):
    """x [rows, cols] -> (codes [rows, pieces * 128], scales).  The scale by trying exponents, the nearest code by searching among all magnitudes."""
    rows = x.shape[0]
    v = _blocks(np.asarray(x, np.float64), squares)
    scale = np.zeros((v.shape[0], v.shape[2]), np.int64)
    codes = np.zeros(v.shape, np.uint8)
    for r, p in np.ndindex(scale.shape):
        block = v[r, :, p]
        if not np.isfinite(block).all():
            scale[r, p] = 255
            continue
        top = np.abs(block).max()
        e = -127
        if top > 0:
            e = max(-127, int(np.floor(np.log2(top))) - 12)
            while top > 448 * 2.0 ** e:
                e += 1
        scale[r, p] = 127 + e
        units = np.abs(np.ldexp(block, -e))
        above = np.searchsorted(GRID, units)                # the first magnitude that is not below
        above = np.minimum(above, 126)
        below = np.maximum(above - 1, 0)
        up, down = GRID[above] - units, units - GRID[below]
        pick = np.where(up < down, above, np.where(up > down, below, np.where(above % 2 == 0, above, below)))
        codes[r, :, p] = pick + 128 * np.signbit(block)
    return codes.reshape(-1, v.shape[2] * 128)[:rows], scale.astype(np.uint8)


def fp8_values(codes, scales, cols):
    """The values that codes and scales stand for, [rows, cols]."""
    codes = np.asarray(codes)
    magnitude = np.append(GRID, np.nan)[codes & 127]
    v = np.where(codes >= 128, -magnitude, magnitude)
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, np.asarray(scales, np.int64) - 127))
    if scales.shape[0] != codes.shape[0]:
        unit = np.repeat(unit, 128, axis=0)[:codes.shape[0]]
    return (v * np.repeat(unit, 128, axis=1))[:, :cols]


def rms_norm(x, residual, gamma, eps):
    """-> (y, sum, rstd)"""
    s = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    rstd = 1.0 / np.sqrt((s * s).mean(axis=1) + eps)
    return s * rstd[:, None] * (1.0 if gamma is None else np.asarray(gamma, np.float64)), s, rstd


def rms_norm_backward(dy, s, rstd, gamma, dsum):
    """-> (dx, dgamma) for a given rstd"""
    dy, s, r = np.asarray(dy, np.float64), np.asarray(s, np.float64), np.asarray(rstd, np.float64)[:, None]
    d = dy * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    dx = r * (d - s * r ** 2 * (d * s).mean(axis=1, keepdims=True))
    return dx + (0.0 if dsum is None else np.asarray(dsum, np.float64)), (dy * s * r).sum(axis=0)


def gated(x, gate, up, act):
    """Values x [rows, k], gate and up [out, k] -> (act(g) u, g, u)"""
    g, u = x @ gate.T, x @ up.T
    return activation(g, act) * u, g, u


def gated_backward(dh, g, u, act):
    """Gradients of the two projections."""
    return dh * u * activation_slope(g, act), dh * activation(g, act)
