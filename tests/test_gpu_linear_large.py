"""Linear layers with millions of rows or with many outputs: every part of the result equals, bit for bit, what a call for that part alone gives.
(A result's sum runs over k in one order, whatever the tile that it is in; the parts' sizes are those of test_gpu_operator_paths.py.)"""

import pytest

from operator_helpers import guarded
from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _parts(count, size):
    """First, last, and two in between that start at no multiple of anything."""
    return [(0, size), (count // 3 + 1, count // 3 + 1 + size), (count // 2 - 7, count // 2 - 7 + size), (count - size, count)]


# 2^22 tiles of 16 x 16 results and more; the last has offsets beyond 32 bits
@pytest.mark.parametrize("rows,k,out,kind,quantised", [(64 * 128 * 128, 64, 1024, "float16", False), (64 * 112 * 112 + 5, 64, 1536, "float16", True),
                                                       (1 << 22, 40, 256, "float32", False), ((1 << 20) + 77, 128, 4100, "bfloat16", False)])
def test_many_short_rows(torch, rows, k, out, kind, quantised):
    dtype = getattr(torch, kind)
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(rows, k, generator=g, device="cuda").to(dtype)
    w = B.patdnn_mxfp4_quantize(torch.randn(out, k, generator=g, device="cuda"))
    bias = torch.randn(out, generator=g, device="cuda")
    scales = None
    if quantised:
        x, scales = B.patdnn_mxfp4_quantize(x)
    y, check = guarded(torch, (rows, out), dtype)
    B.patdnn_mxfp4_linear(x, *w, bias, y, x_scales=scales, act="silu")
    torch.cuda.synchronize()
    check()
    for a, b in _parts(rows, 8200):
        part = B.patdnn_mxfp4_linear(x[a:b], *w, bias, x_scales=None if scales is None else scales[a:b], act="silu", dtype=dtype)
        assert torch.equal(y[a:b], part), (a, b)


def test_many_outputs(torch):
    rows, k, out = 8192, 4096, 151936
    g = torch.Generator(device="cuda").manual_seed(9)
    x, scales = B.patdnn_mxfp4_quantize(torch.randn(rows, k, generator=g, device="cuda"))
    w, w_scales = B.patdnn_mxfp4_quantize(torch.randn(out, k, generator=g, device="cuda"))
    y, check = guarded(torch, (rows, out), torch.bfloat16)
    B.patdnn_mxfp4_linear(x, w, w_scales, None, y, x_scales=scales)
    torch.cuda.synchronize()
    check()
    for a, b in _parts(out, 4096):
        assert torch.equal(y[:, a:b], B.patdnn_mxfp4_linear(x, w[a:b], w_scales[a:b], x_scales=scales, dtype=torch.bfloat16)), (a, b)


# every number of pieces with every number of rows a wavefront: work is sets of 64 rows times sets of 64 outputs, up to 1024, and from 8192 on with 32 sets of outputs
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,out", [(8200, 65), (8200, 1025), (16400, 2050)])
@pytest.mark.parametrize("k", [100, 200, 300, 500])
def test_short_rows_are_exact_where_sums_are(torch, rows, k, out, kind):
    """Small whole numbers: every sum is exact, so results are equal to the product."""
    g = torch.Generator(device="cuda").manual_seed(10)
    x, w = (torch.randint(-3, 4, (count, k), generator=g, device="cuda").float() for count in (rows, out))
    x[:, ::32], w[:, ::32] = 4, 4                              # units of 1 in every block
    want = (x.double() @ w.double().t().contiguous()).float()
    codes = B.patdnn_mxfp4_quantize(w)
    x = x.to(getattr(torch, kind))
    y, check = guarded(torch, (rows, out), torch.float32)
    assert torch.equal(B.patdnn_mxfp4_linear(x, *codes, out=y), want)
    check()
    xc, xs = B.patdnn_mxfp4_quantize(x)
    assert torch.equal(B.patdnn_mxfp4_linear(xc, *codes, x_scales=xs, act="relu"), want.relu())
