"""What the group norm makes of given statistics, to the last bits: against the definition in 64 bits with the mean and the reciprocal deviation that the
call itself returned, so that only the roundings between x and y count.

z = (x - mean) * (rstd * gamma) + beta takes four roundings, each of at most 2^-24 of what it rounds: the difference, the product of the two constants
(both relative to the first term), the sum.  So 4 * 2^-24 of |first term| + |beta|, and with ReLU's own order of operations no more.  SiLU's slope is at
most 1.1; its exponential is taken of z log2(e), rounded, which moves it by 2^-24 |z| of itself, as a rounding of z does; its three further operations
round by 2^-24 (the exponential and the reciprocal by twice that) of the result: 8 * 2^-24 of it.  16-bit types: and half a spacing of y."""

import numpy as np
import pytest

from operator_helpers import U, doubles, types
from oracle import operators as oo
from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


# held (a lane's channels of one group, of several) and in two launches
@pytest.mark.parametrize("shape", [(2, 300, 64, 8), (2, 300, 36, 12), (1, 20000, 16, 8)])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("far,kind", [(0.0, "f32"), (30.0, "f32"), (300.0, "f32"), (3000.0, "f32"), (0.0, "f16"), (300.0, "f16"), (0.0, "bf16"), (30.0, "bf16")])
def test_roundings_between_x_and_y(torch, shape, act, far, kind):
    n, pixels, c, groups = shape
    g = torch.Generator(device="cuda").manual_seed(int(far) + c)
    x = (torch.randn(n, pixels, c, generator=g, device="cuda") + far).to(types(torch)[kind])
    gamma, beta = torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")
    y, mean, rstd = B.patdnn_group_norm(x, groups, gamma, beta, act=act)
    per = lambda t: np.repeat(doubles(t), c // groups, axis=1)[:, None, :]     # noqa: E731
    first = (doubles(x) - per(mean)) * per(rstd) * doubles(gamma)
    z = first + doubles(beta)
    want = oo.activation(z, act)
    allowed = 4 * U["f32"] * (np.abs(first) + np.abs(doubles(beta)))
    if act == "silu":
        allowed = 1.1 * allowed + U["f32"] * (8 + np.abs(z)) * np.abs(want)
    allowed = allowed * 1.01 + 1e-37
    if kind != "f32":
        allowed = allowed + U[kind] * np.abs(want) * 1.01 + 2.0 ** -25
    worst = (np.abs(doubles(y) - want) / allowed).max()
    assert worst <= 1, worst


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("pixels,groups", [(256, 4), (4096, 8), (16384, 8)])
def test_a_plane_of_one_value(torch, kind, act, pixels, groups):
    """A power of two of values that are equal, and exact in every type: their sums and so the mean are exact, and y is the activation of beta."""
    c = 16
    x = torch.full((2, pixels, c), 80.0, device="cuda").to(types(torch)[kind])
    gamma, beta = torch.linspace(0.7, 3.3, c, device="cuda"), torch.linspace(-2, 2, c, device="cuda")
    y, mean, _ = B.patdnn_group_norm(x, groups, gamma, beta, act=act)
    assert bool((mean == 80).all())
    want = oo.activation(doubles(beta), act)
    assert (np.abs(doubles(y) - want) <= 12 * U["f32"] * np.abs(want) + (U[kind] * np.abs(want) * 1.01 if kind != "f32" else 0) + 1e-37).all()
