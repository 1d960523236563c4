"""Group norm on the GPU against the oracle in 64 bits.

Tolerances.  fp32: the rounding errors of a group's M terms add up like a random walk, sqrt(M) 2^-24 of their size, below
4e-6 for the M <= 4096 pixels of a lane and less where lanes join, so 1e-5 of the largest output; a mean that
lies `far` deviations away loses that many times more in x - mean.  dx is a difference that cancels (all of it in a group of one value,
all but eps's share in a group of two): 1e-5 of the largest sum of its terms' magnitudes.  16-bit types: that, and half a spacing of the output.
Sums of gradients (dgamma, dbeta): 1e-5 of the square root of the terms' squares summed times sqrt(terms), which bounds their sizes' sum."""

import numpy as np
import pytest

from oracle import operators as oo
from operator_helpers import U, doubles, guarded, replays, stored, types
from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu
TOL = 1e-5


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _near(got, want, kind, far=0.0, scale=None):
    scale = np.abs(want).max() if scale is None else scale
    allowed = TOL * (1 + far) * scale + (U[kind] * np.abs(want) * 1.01 + 2.0 ** -24 if kind != "f32" else 0)
    worst = (np.abs(got - want) - allowed).max()
    assert worst <= 0, (worst, scale)


def _terms(dy, x, mean, rstd, groups, gamma):
    """The largest sum of magnitudes that an element of dx is a difference of."""
    n, c = x.shape[0], x.shape[-1]
    per = lambda t: np.repeat(np.asarray(t, np.float64), c // groups, axis=1)[:, None, :]      # noqa: E731
    over = lambda t: per(t.reshape(n, -1, groups, c // groups).mean(axis=(1, 3)))              # noqa: E731
    x, g = x.reshape(n, -1, c), 1.1 * np.abs(dy.reshape(n, -1, c) * gamma)
    xh = np.abs((x - per(mean)) * per(rstd))
    return (per(rstd) * (g + over(g) + xh * over(g * xh))).max()


# n, pixels, channels, groups: one value a group, one pixel, one group, one channel a group, three and five channels a group (runs cross groups),
# more channels than a chunk in one group and in several, chunks that end inside the channels, many slabs
SHAPES = [(1, 1, 1, 1), (3, 1, 8, 4), (2, 5, 7, 7), (1, 33, 96, 32), (2, 49, 512, 32), (1, 300, 40, 8), (2, 64, 600, 1), (1, 70, 1030, 2),
          (2, 31, 799, 1), (2, 40, 768, 3), (1, 4000, 16, 4), (4, 129, 48, 48), (1, 2000, 3, 1), (70, 9, 260, 65), (1, 9, 272, 272), (2, 37, 992, 32)]


def _case(torch, shape, kind, seed=3, far=0.0):
    n, pixels, c, groups = shape
    rng = np.random.default_rng([seed, *shape])
    x = stored(torch, rng.standard_normal((n, pixels, c)) * np.exp(rng.standard_normal(c) * 0.3) + rng.standard_normal(c) + far, kind)
    gamma, beta = (rng.standard_normal(c).astype(np.float32) for _ in range(2))
    dy = stored(torch, rng.standard_normal((n, pixels, c)), kind)
    return x, dy, gamma, beta


def _both(torch, shape, kind, act, eps=1e-5, far=0.0):
    n, pixels, c, groups = shape
    x, dy, gamma, beta = _case(torch, shape, kind, far=far)
    # ReLU's gradient jumps where z is 0: the sign of a z within rounding of 0 is nobody's
    y, mean, rstd = oo.group_norm(doubles(x), groups, gamma, beta, eps, "none")
    if act == "relu":
        dy = torch.where(torch.from_numpy(np.abs(y) < 1e-4 * (1 + far)).view(dy.shape), torch.zeros_like(dy), dy)
    y = oo.activation(y, act)
    out, check = guarded(torch, tuple(x.shape), x.dtype)
    g, b = (torch.from_numpy(t).cuda() for t in (gamma, beta))
    got, gm, gr = B.patdnn_group_norm(x.cuda(), groups, g, b, out, eps=eps, act=act)
    torch.cuda.synchronize()
    check()
    _near(doubles(got), y, kind, far)
    assert np.abs(doubles(gm) - mean).max() <= TOL * (1 + far)
    assert (np.abs(doubles(gr) - rstd) <= TOL * (1 + far) * rstd).all()
    dx, check = guarded(torch, tuple(x.shape), x.dtype)
    m32, r32 = mean.astype(np.float32), rstd.astype(np.float32)
    want, wg, wb = oo.group_norm_backward(doubles(dy), doubles(x), m32, r32, groups, gamma, beta, act)
    _, dgamma, dbeta = B.patdnn_group_norm_backward(dy.cuda(), x.cuda(), torch.from_numpy(m32).cuda(), torch.from_numpy(r32).cuda(), groups, g, b, dx, act=act)
    torch.cuda.synchronize()
    check()
    _near(doubles(dx), want, kind, far, _terms(doubles(dy), doubles(x), m32, r32, groups, gamma))
    count = n * pixels
    xh = np.abs((doubles(x) - np.repeat(m32, c // groups, 1)[:, None]) * np.repeat(r32, c // groups, 1)[:, None])
    size = np.abs(doubles(dy)).reshape(count, c) * 1.1
    assert (np.abs(doubles(dbeta) - wb) <= TOL * (1 + far) * np.sqrt(count * (size ** 2).sum(0)) + 1e-30).all()
    assert (np.abs(doubles(dgamma) - wg) <= TOL * (1 + far) * np.sqrt(count * ((size * xh.reshape(count, c)) ** 2).sum(0)) + 1e-30).all()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(torch, shape, kind):
    _both(torch, shape, kind, "silu")


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_activations(torch, act, kind):
    _both(torch, (3, 200, 64, 8), kind, act)


def test_far_from_zero(torch):
    """Values whose mean is 300 times their spread keep their variance."""
    _both(torch, (2, 500, 32, 4), "f32", "none", far=300.0)


def test_eps(torch):
    _both(torch, (2, 20, 16, 4), "f32", "relu", eps=0.5)
    x = torch.full((1, 6, 8), 3.0, device="cuda")
    y, mean, rstd = B.patdnn_group_norm(x, 2, eps=1e-5)
    assert bool((y == 0).all()) and bool((mean == 3).all()) and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5))


@pytest.mark.parametrize("wide,offset", [(100, 0), (131, 5), (104, 8), (98, 2)])
@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_slices_of_wider_tensors(torch, wide, offset, kind):
    n, h, w, c, groups = 2, 6, 7, 96, 32
    x, dy, gamma, beta = _case(torch, (n, h * w, c, groups), kind)
    x, dy = x.view(n, h, w, c), dy.view(n, h, w, c)
    part = slice(offset, offset + c)
    wx, wdy, wy = (torch.full((n, h, w, wide), 9.0, dtype=x.dtype, device="cuda") for _ in range(3))
    wx[..., part], wdy[..., part] = x.cuda(), dy.cuda()
    g, b = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
    y, mean, rstd = B.patdnn_group_norm(wx[..., part], groups, g, b, wy[..., part], act="silu")
    assert bool((wy[..., :offset] == 9).all()) and bool((wy[..., offset + c:] == 9).all())
    _near(doubles(y), oo.group_norm(doubles(x), groups, gamma, beta, 1e-5, "silu")[0], kind)
    wy.fill_(9)
    dx, dgamma, dbeta = B.patdnn_group_norm_backward(wdy[..., part], wx[..., part], mean, rstd, groups, g, b, wy[..., part], act="silu")
    assert bool((wy[..., :offset] == 9).all()) and bool((wy[..., offset + c:] == 9).all())
    want = oo.group_norm_backward(doubles(dy), doubles(x), doubles(mean), doubles(rstd), groups, gamma, beta, "silu")
    _near(doubles(dx), want[0], kind)


def test_broadcast_gradient(torch):
    """The gradient of a sum: one value for all, strides of zero between pixels and images."""
    x = torch.randn(3, 5, 4, 32, device="cuda")
    _, mean, rstd = B.patdnn_group_norm(x, 4)
    one = torch.randn(32, device="cuda").expand(3, 5, 4, 32)
    a = B.patdnn_group_norm_backward(one, x, mean, rstd, 4)
    b = B.patdnn_group_norm_backward(one.contiguous(), x, mean, rstd, 4)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_what_is_not_finite_stays_in_its_group(torch):
    n, pixels, c, groups = 2, 50, 24, 6
    x = torch.randn(n, pixels, c, device="cuda")
    want, _, _ = B.patdnn_group_norm(x, groups, act="relu")
    for value in (float("nan"), float("inf"), float("-inf")):
        bad = x.clone()
        bad[1, 17, 9] = value
        y, _, _ = B.patdnn_group_norm(bad, groups, act="relu")
        hit = torch.zeros_like(y, dtype=torch.bool)
        hit[1, :, 8:12] = True
        assert bool(y[hit].isnan().all()) and torch.equal(y[~hit], want[~hit])


def test_results_repeat_and_nothing_is_added_to(torch):
    x, dy = (torch.randn(4, 700, 64, device="cuda") for _ in range(2))
    work = torch.full((B.patdnn_group_norm_workspace_floats(4, 700, 64, 8, backward=True),), float("nan"), device="cuda")
    front = torch.full((B.patdnn_group_norm_workspace_floats(4, 700, 64, 8),), float("nan"), device="cuda")
    y, mean, rstd = B.patdnn_group_norm(x, 8, act="silu", workspace=front)
    a = B.patdnn_group_norm_backward(dy, x, mean, rstd, 8, act="silu", workspace=work)
    a = [t.clone() for t in a]
    for _ in range(3):
        z = B.patdnn_group_norm(x, 8, act="silu")
        b = B.patdnn_group_norm_backward(dy, x, mean, rstd, 8, act="silu", dgamma=torch.full((64,), 7.0, device="cuda"))
        assert torch.equal(y, z[0]) and all(torch.equal(p, q) for p, q in zip(a, b))


def test_the_two_passes_agree_about_relu(torch):
    """Where the forward pass gave 0 the gradient that reaches the sums is 0: with dy = 1 dbeta counts the positive outputs."""
    x = torch.randn(2, 3000, 32, device="cuda")
    gamma, beta = torch.randn(32, device="cuda"), torch.randn(32, device="cuda")
    y, mean, rstd = B.patdnn_group_norm(x, 4, gamma, beta, act="relu")
    _, _, dbeta = B.patdnn_group_norm_backward(torch.ones_like(x), x, mean, rstd, 4, gamma, beta, act="relu")
    assert torch.equal(dbeta, (y > 0).sum(dim=(0, 1)).float())


def test_no_images(torch):
    x = torch.empty(0, 4, 4, 16, device="cuda")
    y, mean, rstd = B.patdnn_group_norm(x, 4)
    assert y.shape == x.shape and mean.shape == (0, 4)
    _, dgamma, dbeta = B.patdnn_group_norm_backward(x, x, mean, rstd, 4, dgamma=torch.ones(16, device="cuda"), dbeta=torch.ones(16, device="cuda"))
    assert not dgamma.any() and not dbeta.any()


def test_offsets_beyond_32_bits(torch):
    n, pixels, c, groups = 2, 40, 32, 4
    whole = torch.zeros((1 << 32) + 65536, dtype=torch.int8, device="cuda").view(torch.bfloat16)
    x, dy, gamma, beta = _case(torch, (n, pixels, c, groups), "bf16")
    strides = (whole.numel() - pixels * c, c, 1)
    far = torch.as_strided(whole, (n, pixels, c), strides)
    far.copy_(x)
    near_y, mean, rstd = B.patdnn_group_norm(far, groups, act="silu")
    assert torch.equal(near_y, B.patdnn_group_norm(x.cuda(), groups, act="silu")[0])
    grads = B.patdnn_group_norm_backward(dy.cuda(), far, mean, rstd, groups, act="silu")
    far.zero_()
    B.patdnn_group_norm(x.cuda(), groups, None, None, far, act="silu")
    assert torch.equal(far, near_y)
    B.patdnn_group_norm_backward(dy.cuda(), x.cuda(), mean, rstd, groups, None, None, far, act="silu")
    assert torch.equal(far, grads[0])
    assert whole[n * pixels * c:-pixels * c].count_nonzero().item() == 0


def test_streams_and_graphs(torch):
    x, dy = (torch.randn(2, 90, 48, device="cuda") for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(2, 6, device="cuda") for _ in range(2))
    dgamma, dbeta = (torch.empty(48, device="cuda") for _ in range(2))
    front = torch.empty(B.patdnn_group_norm_workspace_floats(2, 90, 48, 6), device="cuda")
    back = torch.empty(B.patdnn_group_norm_workspace_floats(2, 90, 48, 6, backward=True), device="cuda")

    def call():
        B.patdnn_group_norm(x, 6, None, None, y, act="silu", mean=mean, rstd=rstd, workspace=front)
        B.patdnn_group_norm_backward(dy, x, mean, rstd, 6, None, None, dx, act="silu", dgamma=dgamma, dbeta=dbeta, workspace=back)
    for got, want in replays(torch, call, lambda: [y, mean, rstd, dx, dgamma, dbeta], lambda i: (x.normal_(), dy.normal_())):
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = B.patdnn_group_norm(x, 6)[0]
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        got = B.patdnn_group_norm(x, 6, stream=stream)[0]
        side.synchronize()
        assert torch.equal(got, want)
