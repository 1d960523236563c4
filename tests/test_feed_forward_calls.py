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
