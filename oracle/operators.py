"""The operators around the convolutions in IEEE double, each its definition written out: change of channel
order, group norm with an activation and its gradients, MXFP4 and the linear layer on it.  Inputs are
what a caller stores (already rounded to their types); results are not rounded."""

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def activation(z, act):
    if act == "relu":
        return np.where(z <= 0, 0.0, z)
    if act == "silu":
        with np.errstate(over="ignore"):
            return z / (1.0 + np.exp(-z))
    return z


def activation_slope(z, act):
    if act == "relu":
        return np.where(z <= 0, 0.0, 1.0)
    if act == "silu":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)


def _groups(x, groups):
    """[n, ..., c] -> [n, pixels, groups, c / groups]"""
    return np.asarray(x, np.float64).reshape(x.shape[0], -1, groups, x.shape[-1] // groups)


def group_norm(x, groups, gamma, beta, eps, act):
    """x [n, ..., c] -> (y, mean [n, groups], rstd [n, groups])"""
    v = _groups(x, groups)
    mean = v.mean(axis=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    rstd = 1.0 / np.sqrt(var + eps)
    xh = (v - mean[:, None, :, None]) * rstd[:, None, :, None]
    z = xh.reshape(x.shape) * np.asarray(gamma, np.float64) + np.asarray(beta, np.float64)
    return activation(z, act), mean, rstd


def group_norm_backward(dy, x, mean, rstd, groups, gamma, beta, act):
    """-> (dx, dgamma, dbeta) for given statistics"""
    shape, c = x.shape, x.shape[-1]
    per = lambda t: np.repeat(np.asarray(t, np.float64), c // groups, axis=1)[:, None, :]      # noqa: E731
    x, dy = (np.asarray(t, np.float64).reshape(shape[0], -1, c) for t in (x, dy))
    gamma, beta = np.asarray(gamma, np.float64), np.asarray(beta, np.float64)
    xh = (x - per(mean)) * per(rstd)
    dz = dy * activation_slope(xh * gamma + beta, act)
    dbeta, dgamma = dz.sum(axis=(0, 1)), (dz * xh).sum(axis=(0, 1))
    g = dz * gamma
    m = x.shape[1] * (c // groups)
    a = per(_groups(g, groups).sum(axis=(1, 3)) / m)
    b = per(_groups(g * xh, groups).sum(axis=(1, 3)) / m)
    return (per(rstd) * (g - a - xh * b)).reshape(shape), dgamma, dbeta


def mxfp4_quantize(x):
    """x [rows, cols] -> (codes, scales) as they are stored.  The nearest code is searched among all eight magnitudes."""
    rows, cols = x.shape
    pieces = -(-cols // 128)
    v = np.zeros((rows, pieces * 128))
    v[:, :cols] = x
    v = v.reshape(rows, pieces * 4, 32)
    top = np.abs(v).max(axis=2)
    bad = ~np.isfinite(v).all(axis=2)
    scale = np.zeros((rows, pieces * 4), np.int64)
    codes = np.zeros(v.shape, np.uint8)
    for r, b in np.ndindex(scale.shape):
        if bad[r, b]:
            scale[r, b] = 255
            continue
        if top[r, b] > 0:
            scale[r, b] = 127 + max(-127, int(np.frexp(top[r, b])[1]) - 1 - 2)
        units = np.ldexp(np.abs(v[r, b]), int(127 - scale[r, b]))
        away = np.abs(units[:, None] - GRID[None, :])
        near = away == away.min(axis=1, keepdims=True)
        # of two nearest codes the even one
        pick = np.where(near.sum(axis=1) == 2, np.argmax(near & (np.arange(8) % 2 == 0), axis=1), np.argmax(near, axis=1))
        codes[r, b] = pick + 8 * np.signbit(v[r, b])
    codes = codes.reshape(rows, -1)
    return (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8), scale.astype(np.uint8)


def mxfp4_values(codes, scales, cols):
    """The values that codes and scales stand for, [rows, cols]."""
    both = np.stack((codes & 15, codes >> 4), axis=2).reshape(codes.shape[0], -1)
    signed = np.where(both >= 8, -1.0, 1.0) * GRID[both & 7]
    unit = np.repeat(np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127)), 32, axis=1)
    return (signed * unit)[:, :cols]


def linear(x, w, bias, act):
    """act(x w^T + bias) for values x [rows, k], w [out, k], and the sums of the magnitudes of its terms"""
    z = x @ w.T
    size = np.abs(x) @ np.abs(w).T
    if bias is not None:
        z = z + bias
        size = size + np.abs(bias)
    return activation(z, act), size
