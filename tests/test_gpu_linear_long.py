"""Linear layers of long rows on small whole numbers: codes hold them exactly and every sum stays below 2^24, so outputs are equal to the product, whatever
the order of the sums, and a block, piece or slice of k that is left out or counted twice shows at any length.  (A bound from the rounding of k additions
grows with k until it holds for anything.)  That it would show is tested on the host, with the mistake in the expected product."""

import numpy as np
import pytest

from operator_helpers import types
from paper_2001_00138_amd import binding as B

# x in the LDS of the workgroups that multiply it, x that does not fit, few rows in codes, tiles of each size, in slices of k and whole;
# k on either side of whole blocks of 32, pieces of 128 and stages of four
CASES = [(1, 25088, 300), (1, 60000, 40), (2, 120000, 40), (9, 25000, 40), (16, 15000, 40), (16, 20000, 40), (3, 300000, 40), (5, 300001, 17), (17, 8193, 70),
         (40, 5000, 520), (70, 9000, 40), (300, 30000, 40), (64, 25088, 300), (65, 25185, 130), (600, 12900, 1030), (40, 4100, 5000)]


def _numbers(rows, k, out):
    rng = np.random.default_rng([31, rows, k, out])
    x, w = (rng.integers(-3, 4, (count, k)).astype(np.float32) for count in (rows, out))
    x[:, ::32], w[:, ::32] = 4, 4                              # units of 1 in every block
    return x, w


@pytest.mark.parametrize("rows,k,out", [c for c in CASES if c[0] * c[1] * c[2] < 3e8])
def test_what_is_left_out_would_show(rows, k, out):
    x, w = _numbers(rows, k, out)
    whole = x @ w.T
    assert np.abs(x).astype(np.float64).max() * np.abs(w).max() * k < 2 ** 24
    for size in (32, 128, 512):
        blocks = range(0, k, size)
        for first in {0, blocks[len(blocks) // 3], blocks[-1]}:
            assert (x[:, first:first + size] @ w[:, first:first + size].T != 0).any()
    for slices in range(2, 17):
        edges = [k * i // slices for i in range(slices + 1)]
        assert all((x[:, a:b] @ w[:, a:b].T != 0).any() for a, b in zip(edges, edges[1:]))
    assert (whole != 0).any()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,k,out", CASES)
def test_equal(rows, k, out, kind):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    x, w = (torch.from_numpy(t).cuda() for t in _numbers(rows, k, out))
    want = (x.double() @ w.double().t().contiguous()).float()
    bias = torch.arange(out, device="cuda", dtype=torch.float32) - out // 2
    codes = B.patdnn_mxfp4_quantize(w)
    x = x.to(types(torch)[kind])
    assert torch.equal(B.patdnn_mxfp4_linear(x, *codes, dtype=torch.float32), want)
    xc, xs = B.patdnn_mxfp4_quantize(x)
    assert torch.equal(B.patdnn_mxfp4_linear(xc, *codes, bias, x_scales=xs), want + bias)
