"""Planes of one value, of any number of pixels: where the sums are exact (small whole numbers) so is the mean, y is beta and the gradient of a sum is 0, also
where 1 / M is no binary fraction and the reciprocal deviation, 1 / sqrt(eps), makes much of what the mean is off by."""

import pytest

from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _check(torch, n, pixels, c, groups, kind, value):
    x = torch.full((n, pixels, c), float(value), device="cuda", dtype=getattr(torch, kind))
    beta = torch.arange(c, device="cuda", dtype=torch.float32) - c // 2
    y, mean, rstd = B.patdnn_group_norm(x, groups, None, beta)
    case = (n, pixels, c, groups, kind, value)
    assert bool((mean == value).all()), case
    assert torch.equal(y, beta.to(x.dtype).expand_as(y)), case
    dx, dgamma, dbeta = B.patdnn_group_norm_backward(torch.ones_like(x), x, mean, rstd, groups)
    assert not dx.any() and not dgamma.any() and bool((dbeta == n * pixels).all()), case


@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("c,groups", [(8, 8), (8, 4), (12, 4), (16, 4), (64, 8), (40, 2)])
def test_small(torch, c, groups, kind):
    for pixels in range(1, 200):
        _check(torch, 2, pixels, c, groups, kind, 3)


@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("n,pixels,c,groups", [(1, 3007, 128, 32), (64, 3007, 64, 8), (70, 197, 64, 2), (600, 61, 48, 12), (2, 12005, 48, 24), (1, 3001, 600, 1), (2, 9001, 3, 1)])
def test_larger(torch, n, pixels, c, groups, kind):
    for value in (3, 80, -7):
        _check(torch, n, pixels, c, groups, kind, value)
