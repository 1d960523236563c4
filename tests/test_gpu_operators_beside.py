"""Outputs beside their inputs in one wider tensor, as a network that concatenates features has them: equal, bit for bit, to outputs of their own."""

import pytest

from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


# held, and in two launches
@pytest.mark.parametrize("pixels", [(7, 9), (100, 150)])
@pytest.mark.parametrize("kind", ["float32", "float16"])
@pytest.mark.parametrize("first", [0, 29])
def test_group_norm(torch, pixels, kind, first):
    c, wide, second = 24, 60, 29 - first
    whole = torch.randn(2, *pixels, wide, device="cuda").to(getattr(torch, kind))
    x, y = whole[..., first:first + c], whole[..., second:second + c]
    gamma, beta = torch.randn(c, device="cuda"), torch.randn(c, device="cuda")
    before = whole.clone()
    want, mean, rstd = B.patdnn_group_norm(x.contiguous(), 3, gamma, beta, act="silu")
    assert torch.equal(B.patdnn_group_norm(x, 3, gamma, beta, y, act="silu")[0], want)
    dy = torch.randn_like(want)
    back = B.patdnn_group_norm_backward(dy, x.contiguous(), mean, rstd, 3, gamma, beta, act="silu")
    got = B.patdnn_group_norm_backward(dy, x, mean, rstd, 3, gamma, beta, y, act="silu")
    assert all(torch.equal(a, b) for a, b in zip(got, back))
    before[..., second:second + c] = y
    assert torch.equal(whole, before)


@pytest.mark.parametrize("rows,k", [(2, 200), (20, 200), (300, 200), (300, 700)])
def test_linear(torch, rows, k):
    out = 70
    whole = torch.randn(rows, k + out + 3, device="cuda").half()
    w = B.patdnn_mxfp4_quantize(torch.randn(out, k, device="cuda"))
    before = whole.clone()
    want = B.patdnn_mxfp4_linear(whole[:, :k].contiguous(), *w)
    y = B.patdnn_mxfp4_linear(whole[:, :k], *w, out=whole[:, k + 1:k + 1 + out])
    assert torch.equal(y, want)
    before[:, k + 1:k + 1 + out] = want
    assert torch.equal(whole, before)
