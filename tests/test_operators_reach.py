"""Sizes that the operators' kernels reach are not refused: a call without tensors is turned down for them, and not for its size.  Nothing is launched."""

import ctypes

import pytest

from paper_2001_00138_amd import binding as B

L = B.lib


@pytest.mark.parametrize("rows,k,out", [
    (64 * 128 * 128, 64, 1024), (64 * 112 * 112, 64, 1536), (1 << 20, 512, 1024), (8192, 4096, 151936), (1 << 22, 40, 64),
    (1 << 20, 1024, 1 << 16), (100000, 300, 50000), (1 << 28, 17, 16), (2 ** 31 - 257, 1, 1),
    (4096, 25088, 1 << 20), (20, 256, (1 << 26) - 32), (1, 256, (1 << 26) - 32)])
@pytest.mark.parametrize("x_type", [B.PATDNN_F32, B.PATDNN_BF16, B.PATDNN_MXFP4])
def test_linear(rows, k, out, x_type):
    d = B.LinearDesc(rows, k, out, x_type, B.PATDNN_F16, 0, k, out)
    assert L().patdnn_mxfp4_linear(ctypes.byref(d), None, None, None, None, None, None, None, 0, None) == B.PATDNN_EINVAL
    assert "NULL" in L().patdnn_last_error().decode()


@pytest.mark.parametrize("rows,k,out", [(1, 256, (1 << 26) + 1), (64, 256, (1 << 26) + 1), (1 << 20, 256, (1 << 26) + 1), (2 ** 31 - 256, 1, 1), (2 ** 31 - 1, 100, 1),
                                        (2 ** 31 - 300, 1025, 1), (1 << 31 - 4, 200000 * 128, 1 << 20)])
def test_linear_beyond(rows, k, out):
    d = B.LinearDesc(rows, k, out, B.PATDNN_F16, B.PATDNN_F16, 0, k, out)
    assert L().patdnn_mxfp4_linear(ctypes.byref(d), None, None, None, None, None, None, None, 0, None) == B.PATDNN_EUNSUPPORTED
    assert L().patdnn_mxfp4_linear_workspace_bytes(ctypes.byref(d)) == 0
