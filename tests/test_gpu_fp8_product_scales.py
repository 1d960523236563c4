"""Products of fp8 codes with scales near both ends of a byte, and all finite codes, subnormal ones among them.

Tolerances as in the tests of ordinary scales.  Besides, sums with fp32's precision (results in fp32, and few rows) take values below 2^-126 as bfloat16's subnormals, whose spacing is
2^-133: at most that for each term's other factor."""

import numpy as np
import pytest

from oracle import feed_forward as ff
from operator_helpers import doubles, types
from paper_2001_00138_amd import binding as B
from test_gpu_fp8_products import KINDS, near, sums_of

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def operand(torch, rng, rows, k, low, high, squares=False):
    """-> (codes, scales with bytes of [low, high], values)"""
    pieces = -(-k // 128)
    codes = rng.integers(0, 256, (rows, pieces * 128)).astype(np.uint8)
    codes[codes % 128 == 127] = 0                        # not a number
    codes[:, k:] = 0
    scales = rng.integers(low, high + 1, (-(-rows // 128) if squares else rows, pieces)).astype(np.uint8)
    scales[0, 0], scales[-1, -1] = low, high
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), ff.fp8_values(codes, scales, pieces * 128)


# (few rows; the tiles of 64; those of 128 and 256)
@pytest.mark.parametrize("rows,k,n", [(1, 700, 50), (12, 300, 200), (40, 1500, 130), (300, 520, 400), (1700, 300, 1600), (4100, 200, 3900)])
@pytest.mark.parametrize("x_bytes,w_bytes", [((0, 20), (230, 246)), ((230, 246), (0, 20)), ((0, 0), (246, 246))])
def test_far_ends(torch, rows, k, n, x_bytes, w_bytes):
    rng = np.random.default_rng([rows, k, *x_bytes])
    xc, xs, x = operand(torch, rng, rows, k, *x_bytes)
    for squares in (False, True):
        (wc, ws, w), (vc, vs, v) = operand(torch, rng, n, k, *w_bytes, squares), operand(torch, rng, n, k, *w_bytes, squares)
        for kind in KINDS:
            (z, off), (y, off2) = sums(x, w, kind), sums(x, v, kind)
            got = B.patdnn_fp8_linear(xc, xs, wc, ws, dtype=types(torch)[kind])
            assert near(doubles(got), z, off, kind)
            both = B.patdnn_fp8_gated_backward(torch.ones(rows, n, device="cuda"), xc, xs, wc, ws, vc, vs, act="none", dtype=types(torch)[kind])
            assert near(doubles(both), np.hstack((y, z)), np.hstack((off2, off)), kind)


def sums(x, w, kind):
    """As sums_of, whose groups of eight are too many for the larger sizes: there the sum of their largest is at most that of all."""
    if x.shape[0] * w.shape[0] < 200000:
        z, off = sums_of(x, w, kind)
    else:
        z, size = x @ w.T, np.abs(x) @ np.abs(w).T
        off = (x.shape[1] * u + (7 * 2.0 ** -13 if kind != "f32" else 0)) * size
    tiny = lambda t: 2.0 ** -133 * (np.abs(t) < 2.0 ** -126)          # noqa: E731
    return z, off + tiny(x) @ np.abs(w).T + np.abs(x) @ tiny(w).T


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_below_the_range_and_beyond_it(torch, rows):
    """Two factors near 2^-127 leave nothing; a value of 2^128, as the lowest value of a type is quantised to, is infinite where sums have fp32's precision."""
    rng = np.random.default_rng(rows)
    xc, xs, _ = operand(torch, rng, rows, 300, 0, 5)
    wc, ws, _ = operand(torch, rng, 200, 300, 0, 5)
    for kind in KINDS:
        assert bool((B.patdnn_fp8_linear(xc, xs, wc, ws, dtype=types(torch)[kind]) == 0).all())
    v = torch.ones(rows, 300)
    v[rows - 1, 200] = torch.finfo(torch.bfloat16).min
    xc, xs = B.patdnn_fp8_quantize(v.cuda())
    wc, ws = B.patdnn_fp8_quantize(torch.full((200, 300), 2.0 ** -20).cuda())
    assert int(xs[rows - 1, 1]) == 247 and bool((B.patdnn_fp8_dequantize(xc, xs, 300)[rows - 1, 200] == -float("inf")).all())
    got = B.patdnn_fp8_linear(xc, xs, wc, ws)
    assert bool((got[rows - 1] == -float("inf")).all()) and bool((got[:rows - 1] == 300 * 2.0 ** -20).all())
