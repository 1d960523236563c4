"""Calls of the feed-forward block's operators at the borders of what their documentation allows: the largest sizes, no rows, gradients that nobody wants."""

import ctypes

import pytest
import torch

from paper_2001_00138_amd import binding as B
from test_feed_forward_binding import _device, library                  # noqa: F401 (a fixture)

P = 1 << 20                   # stands for device addresses that no call gets as far as reading


def test_codes_of_no_rows_transposed(library):                           # noqa: F811
    """What the call of no rows returned may be given back to it, in either layout."""
    x = _device(torch.zeros(0, 256))
    for blocks in ("rows", "squares"):
        codes, scales = B.patdnn_fp8_quantize(x, blocks=blocks, transposed=True)
        assert codes.shape == (256, 0)
        assert B.patdnn_fp8_quantize(x, codes, scales, blocks=blocks, transposed=True)[0] is codes
    assert len(library.calls) == 4


def test_norm_backward_without_the_gradient_of_gamma(library):           # noqa: F811
    """dgamma=False: no partial sums, no workspace, no second launch."""
    x, r = _device(torch.zeros(3, 256)), _device(torch.zeros(3))
    seen = []
    run = library.__getattr__("patdnn_rms_norm_backward")

    def call(*args):
        seen.append(args)
        return run(*args) if args[-4] else B.PATDNN_OK
    library.patdnn_rms_norm_backward = call
    dx, dgamma = B.patdnn_rms_norm_backward(x, x, r, dgamma=False)
    assert dx.shape == x.shape and dgamma is None and seen[0][-4] is None and seen[0][-3] is None and seen[0][-2] == 0
    gamma = _device(torch.zeros(256))
    assert B.patdnn_rms_norm_backward(x, x, r, gamma, dgamma=False, workspace=_device(torch.zeros(9)))[1] is None and seen[1][-4] is None
    assert B.patdnn_rms_norm_backward(x, x, r, gamma)[1].shape == (256,) and seen[2][-4]


def _border(call, last, first, *rest):
    """The last size is taken (and refused for a NULL pointer alone), the first beyond it is not."""
    for desc, status, word in ((last, B.PATDNN_EINVAL, "NULL"), (first, B.PATDNN_EUNSUPPORTED, "large")):
        assert call(ctypes.byref(desc), *rest) == status and word in B.lib().patdnn_last_error().decode()


# 16, 32 and 64 threads a row, 256 in a workgroup; 8 to 32 columns a thread beyond
@pytest.mark.parametrize("cols,rows", [(1, 2 ** 28 - 16), (128, 2 ** 28 - 16), (129, 2 ** 27 - 8), (512, 2 ** 26 - 4), (513, 2 ** 24 - 1), (4096, 2 ** 23 - 1),
                                       (8192, 2 ** 22 - 1), (40000, 2 ** 22 - 1)])
def test_most_rows_of_a_norm(cols, rows):
    desc = lambda n: B.RmsDesc(n, cols, 2, 2, 1e-6, cols, cols, cols, cols)      # noqa: E731
    _border(B.lib().patdnn_rms_norm, desc(rows), desc(rows + 1), None, None, None, None, P, None, None, None)


@pytest.mark.parametrize("name,args", [("linear", 6), ("gated", 8), ("gated_backward", 9)])
def test_largest_products(name, args):
    call, room = getattr(B.lib(), f"patdnn_fp8_{name}"), getattr(B.lib(), f"patdnn_fp8_{name}_workspace_bytes")
    desc = lambda rows, k, n: B.Fp8Desc(rows, k, n, 0, 2, 0, 2, n, n)             # noqa: E731
    nothing = [None] * args + [None, 0, None]
    for rows in (1, 8, 9, 16):
        _border(call, desc(rows, 128, 2 ** 26 - 16), desc(rows, 128, 2 ** 26 - 15), *nothing)
    # 2^22 - 1 = 3 * 1398101 tiles of 64 x 64
    _border(call, desc(1398101 * 64, 128, 192), desc(1398101 * 64 + 1, 128, 192), *nothing)
    _border(call, desc(64 * (2 ** 22 - 1), 128, 64), desc(64 * (2 ** 22 - 1) + 1, 128, 64), *nothing)
    # rows too long for the tiles' offsets
    _border(call, desc(16 * (2 ** 22 - 1), 8388481, 16), desc(16 * (2 ** 22 - 1) + 1, 8388481, 16), *nothing)
    assert room(ctypes.byref(desc(16, 128, 2 ** 26 - 15))) == 0


def test_most_outputs_of_a_layer_of_four_bits():
    desc = lambda n: B.LinearDesc(3, 32, n, 3, 2, 0, 0, n)                        # noqa: E731
    assert B.lib().patdnn_mxfp4_linear(ctypes.byref(desc(2 ** 26 - 15)), *[P] * 7, 0, None) == B.PATDNN_EUNSUPPORTED
    assert B.lib().patdnn_mxfp4_linear(ctypes.byref(desc(2 ** 26 - 16)), *[None] * 7, 0, None) == B.PATDNN_EINVAL
