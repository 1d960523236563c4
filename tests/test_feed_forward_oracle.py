"""oracle/feed_forward.py against routes of its own: torch's conversions, differences, hand-made blocks."""

import numpy as np
import pytest
import torch

from oracle import feed_forward as ff


def test_grid_is_torchs():
    codes = torch.arange(127, dtype=torch.uint8)
    assert (codes.view(torch.float8_e4m3fn).double().numpy() == ff.GRID).all() and ff.GRID[-1] == 448


@pytest.mark.parametrize("squares", [False, True])
def test_codes_are_torchs(squares):
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((140, 300)) * np.exp(rng.standard_normal((140, 1)) * 3)).astype(np.float32)
    codes, scales = ff.fp8_quantize(x, squares)
    assert codes.shape == (140, 384) and scales.shape == ((2 if squares else 140), 3)
    unit = np.repeat(np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 128 if squares else 1, axis=0)[:140], 128, axis=1)[:, :300]
    want = torch.from_numpy((x / unit).astype(np.float32)).to(torch.float8_e4m3fn)        # the division is exact
    assert (want.view(torch.uint8).numpy() == codes[:, :300]).all() and not codes[:, 300:].any()
    assert (ff.fp8_values(codes, scales, 300) == want.double().numpy() * unit).all()
    for r in range(scales.shape[0]):
        for p in range(3):
            top = np.abs(x[r * 128:r * 128 + 128, p * 128:p * 128 + 128] if squares else x[r, p * 128:p * 128 + 128]).max()
            e = int(scales[r, p]) - 127
            assert 224 * 2.0 ** e < top <= 448 * 2.0 ** e


def test_blocks_by_hand():
    x = np.zeros((5, 128))
    x[0, 0], x[1, 0], x[2, 0], x[3, 3], x[4, 5] = 448, np.nextafter(448, 500), 2.0 ** -149, np.inf, -464
    codes, scales = ff.fp8_quantize(x)
    assert scales[:, 0].tolist() == [127, 128, 0, 255, 128]
    assert codes[0, 0] == 126 and codes[3].max() == 0 and codes[4, 5] == 128 + 0x76 + 0        # -232 units of 2: -232 lies between 224 and 240
    assert np.isnan(ff.fp8_values(codes, scales, 128)[3]).all()


def test_norm_gradients_by_differences():
    rng = np.random.default_rng(5)
    x, res, gamma, dy = rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal((3, 7))
    _, s, rstd = ff.rms_norm(x, res, gamma, 1e-3)
    dx, dgamma = ff.rms_norm_backward(dy, s, rstd, gamma, np.ones((3, 7)))
    f = lambda x, g: (ff.rms_norm(x, res, g, 1e-3)[0] * dy).sum()      # noqa: E731
    h = 1e-6
    for i in np.ndindex(3, 7):
        e = np.zeros((3, 7))
        e[i] = h
        assert abs((f(x + e, gamma) - f(x - e, gamma)) / (2 * h) + 1 - dx[i]) < 1e-8
    for i in range(7):
        e = np.zeros(7)
        e[i] = h
        assert abs((f(x, gamma + e) - f(x, gamma - e)) / (2 * h) - dgamma[i]) < 1e-8


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_gated_gradients_by_differences(act):
    rng = np.random.default_rng(6)
    g, u, dh = rng.standard_normal((4, 5)) * 3, rng.standard_normal((4, 5)), rng.standard_normal((4, 5))
    eye = np.eye(5)
    dg, du = ff.gated_backward(dh, g, u, act)
    f = lambda g, u: ff.gated(np.concatenate((g, u), 1), np.hstack((eye, 0 * eye)), np.hstack((0 * eye, eye)), act)[0]      # noqa: E731
    h = 1e-6
    assert np.abs((f(g + h, u) - f(g - h, u)) / (2 * h) * dh - dg).max() < 1e-8
    assert np.abs((f(g, u + h) - f(g, u - h)) / (2 * h) * dh - du).max() < 1e-8
