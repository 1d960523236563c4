"""The norm's backward pass for a gamma that is frozen or not there: the same gradient of the rows, and nothing else."""

import pytest

from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


# (rows that share a workgroup, rows held with one run a lane and with two, rows read twice)
@pytest.mark.parametrize("rows,cols", [(0, 64), (300, 100), (70, 3000), (5, 9000), (3, 40000)])
def test_rows_gradient_alone(torch, rows, cols):
    torch.manual_seed(cols)
    s, dy, dsum = (torch.randn(rows, cols, device="cuda").bfloat16() for _ in range(3))
    gamma = torch.rand(cols, device="cuda")
    rstd = B.patdnn_rms_norm(s)[3]
    for g in (None, gamma):
        want, dgamma = B.patdnn_rms_norm_backward(dy, s, rstd, g, dsum=dsum)
        got, none = B.patdnn_rms_norm_backward(dy, s, rstd, g, dsum=dsum, dgamma=False)
        assert none is None and dgamma.shape == (cols,) and torch.equal(got, want)
