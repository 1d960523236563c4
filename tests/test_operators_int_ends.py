"""Sizes at the end of a C int: a count that the kernels' 32-bit sums would carry past it is refused, and what is just below is planned in earnest.
Nothing is launched."""

import ctypes

import pytest

from paper_2001_00138_amd import binding as B

L = B.lib
P = 1 << 20                        # stands for device addresses that no call gets as far as reading
Q, R, S, T = P << 24, P << 25, P << 26, P << 27
MOST = 2 ** 31 - 1025              # pixels of a group norm


def _norm(n, pixels, c, groups, kind):
    image = pixels * c
    return ctypes.byref(B.NormDesc(n, pixels, c, groups, kind, 0, 1e-5, image, c, image, c, image, c))


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("n,pixels,c,groups", [
    (n, pixels, c, groups) for n in (1, 3) for pixels in (2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 30, 2 ** 31 - 40, 2 ** 31 - 1000, MOST + 1) for c, groups in ((1, 1), (3, 1), (16, 2))
] + [(n, pixels, c, 1) for n in (1, 3) for pixels in (1, 2) for c in (2 ** 31 - 1, 2 ** 31 - 8, MOST + 1)] + [(1, 1, 2 ** 31 - 1, 2 ** 31 - 1)])
def test_norm_too_long(n, pixels, c, groups, kind):
    d = _norm(n, pixels, c, groups, kind)
    for backward in (0, 1):
        assert L().patdnn_group_norm_workspace_floats(d, backward) == 0
    assert L().patdnn_group_norm(d, P, None, None, Q, None, None, R, 1 << 62, None) == B.PATDNN_EUNSUPPORTED
    assert "large" in L().patdnn_last_error().decode()
    assert L().patdnn_group_norm_backward(d, S, P, T, T, None, None, Q, None, None, R, 1 << 62, None) == B.PATDNN_EUNSUPPORTED
    assert "large" in L().patdnn_last_error().decode()


@pytest.mark.parametrize("pixels,c,groups", [(pixels, c, groups) for pixels in (MOST, MOST - 1, 2 ** 31 - 2 ** 24, 2 ** 31 - 2 ** 23 + 1, 2 ** 30 + 1)
                                             for c, groups in ((1, 1), (3, 1), (16, 2))] +
                         [(1, (1 << 27) + 1, 1), (2, 1 << 27, 1), (1, 8191 << 14, 1 << 14)])
@pytest.mark.parametrize("kind", [0, 1])
def test_norm_as_long_as_it_goes(pixels, c, groups, kind):
    d = _norm(1, pixels, c, groups, kind)
    for backward in (0, 1):
        floats = L().patdnn_group_norm_workspace_floats(d, backward)
        # per slab, of which an image has up to 128, two sums a group and chunk of 256 channels, or a channel
        assert 0 < floats <= 128 * 2 * (c if backward else groups * -(-(c // groups) // 256)), (backward, floats)
        out = (ctypes.c_int32 * 8)()
        assert L().patdnn_internal_norm_plan(d, backward, out) == B.PATDNN_OK
        assert out[0] == 0                                 # nothing of that size is held in registers


@pytest.mark.parametrize("rows", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 15, 2 ** 31 - 16, 2 ** 31 - 100, 2 ** 28])
@pytest.mark.parametrize("cols", [1, 128, 129, 2048, 2049])
def test_quantise_too_many_rows(rows, cols):
    """No rows of memory but the first: a row for all to quantise, of strides of zero."""
    assert L().patdnn_mxfp4_quantize(P, 0, rows, cols, 0, 1 << 50, 1 << 51, None) == B.PATDNN_EUNSUPPORTED
    assert "large" in L().patdnn_last_error().decode()
    assert L().patdnn_mxfp4_dequantize(1 << 50, 1 << 51, rows, cols, P, 1, cols, None) == B.PATDNN_EUNSUPPORTED
    assert "large" in L().patdnn_last_error().decode()
