"""Calls of the feed-forward block's operators at the borders of what their documentation allows: the largest sizes, no rows, gradients that nobody wants."""

import ctypes

import torch

from paper_2001_00138_amd import binding as B
from test_feed_forward_binding import OnDevice, _device, library        # noqa: F401 (a fixture)


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
