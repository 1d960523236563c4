"""The oracle of the operators around the convolutions against routes that share nothing with it: torch in float64,
differences for the gradients, hand-worked codes."""

import numpy as np
import pytest
import torch

from oracle import operators as oo

ACTS = {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu}


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("n,pixels,c,groups", [(1, 1, 4, 2), (2, 7, 6, 3), (3, 5, 8, 1), (2, 9, 5, 5)])
def test_group_norm_is_torchs(act, n, pixels, c, groups):
    rng = np.random.default_rng(5)
    x, gamma, beta = rng.standard_normal((n, pixels, c)) + 3, rng.standard_normal(c), rng.standard_normal(c)
    y, mean, rstd = oo.group_norm(x, groups, gamma, beta, 1e-3, act)
    t = torch.from_numpy(x).transpose(1, 2).requires_grad_()
    g, b = torch.from_numpy(gamma).requires_grad_(), torch.from_numpy(beta).requires_grad_()
    want = ACTS[act](torch.nn.functional.group_norm(t, groups, g, b, 1e-3))
    assert np.abs(y - want.detach().transpose(1, 2).numpy()).max() < 1e-12
    dy = rng.standard_normal(y.shape)
    want.backward(torch.from_numpy(dy).transpose(1, 2))
    dx, dgamma, dbeta = oo.group_norm_backward(dy, x, mean, rstd, groups, gamma, beta, act)
    assert np.abs(dx - t.grad.transpose(1, 2).numpy()).max() < 1e-10
    assert np.abs(dgamma - g.grad.numpy()).max() < 1e-11 and np.abs(dbeta - b.grad.numpy()).max() < 1e-11


@pytest.mark.parametrize("act", ["none", "silu"])
def test_gradients_are_the_differences(act):
    rng = np.random.default_rng(6)
    x, gamma, beta = rng.standard_normal((2, 5, 6)), rng.standard_normal(6), rng.standard_normal(6)
    dy = rng.standard_normal(x.shape)
    loss = lambda x, g, b: (oo.group_norm(x, 2, g, b, 1e-5, act)[0] * dy).sum()        # noqa: E731
    _, mean, rstd = oo.group_norm(x, 2, gamma, beta, 1e-5, act)
    grads = oo.group_norm_backward(dy, x, mean, rstd, 2, gamma, beta, act)
    args = [x, gamma, beta]
    h = 1e-6
    for k in range(3):
        for i in np.ndindex(args[k].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[k][i] += h
            down[k][i] -= h
            # second-order differences of a function of size 10: h^2 and rounding / h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grads[k][i]) < 1e-7


def test_mxfp4_by_hand():
    x = np.zeros((2, 40), np.float32)
    # largest 7: units of 2^(2-2) = 1; ties 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4; 7 -> 6
    x[0, :10] = [7, 0.25, 0.75, -1.25, 1.75, -2.5, 3.5, 5, 5.01, -0.0]
    x[0, 32:35] = [0.375, -0.09375, 0.1]             # largest 0.375 = 6 units of 2^-4; 1.5; 1.6 -> 1.5
    x[1, 3] = np.inf
    codes, scales = oo.mxfp4_quantize(x)
    assert codes.shape == (2, 64) and scales.tolist() == [[127, 123, 0, 0], [255, 0, 0, 0]]
    unpacked = np.stack((codes & 15, codes >> 4), axis=2).reshape(2, -1)
    assert unpacked[0, :10].tolist() == [7, 0, 2, 8 + 2, 4, 8 + 4, 6, 6, 7, 8]
    assert unpacked[0, 32:35].tolist() == [7, 8 + 3, 3] and not unpacked[1].any()
    values = oo.mxfp4_values(codes, scales, 40)
    assert values[0, :9].tolist() == [6, 0, 1, -1, 2, -2, 4, 4, 6] and values[0, 32:35].tolist() == [0.375, -0.09375, 0.09375]
    assert np.isnan(values[1, :32]).all() and not values[1, 32:].any()


def test_mxfp4_keeps_what_it_holds():
    rng = np.random.default_rng(8)
    values = rng.choice(np.concatenate((oo.GRID, -oo.GRID)), (5, 256)) * np.repeat(np.exp2(rng.integers(-20, 20, (5, 8))), 32, axis=1)
    values[:, ::32] = 6 * np.exp2(rng.integers(21, 25, (5, 8)))          # the scale is the one that 6 units have
    kept = oo.mxfp4_values(*oo.mxfp4_quantize(values.astype(np.float32)), 256)
    again = oo.mxfp4_values(*oo.mxfp4_quantize(kept.astype(np.float32)), 256)
    assert (kept == again).all()


def test_mxfp4_extremes():
    big, tiny = np.float32(3.4e38), np.float32(1e-45)
    codes, scales = oo.mxfp4_quantize(np.array([[big] + [0] * 31 + [tiny] + [0] * 31], np.float32))
    assert scales[0, :2].tolist() == [127 + 127 - 2, 0]
    assert codes[0, 0] == 7 and codes[0, 16] == 0


def test_linear_is_a_product():
    rng = np.random.default_rng(9)
    x, w, b = rng.standard_normal((3, 20)), rng.standard_normal((4, 20)), rng.standard_normal(4)
    y, size = oo.linear(x, w, b, "silu")
    z = torch.nn.functional.linear(*(torch.from_numpy(t) for t in (x, w, b)))
    assert np.abs(y - torch.nn.functional.silu(z).numpy()).max() < 1e-13
    assert (size >= np.abs(z.numpy())).all()
