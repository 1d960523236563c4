"""Root-mean-square norm of rows whose squares pass fp32's range though their mean does not, and of rows whose squares fall below it though the root of their mean does not.

Tolerances as in the tests of ordinary rows: powers of two that a row is scaled by have no rounding, and squares that fall below fp32's smallest are less than 2^-40 of the sum."""

import numpy as np
import pytest

from oracle import feed_forward as ff
from operator_helpers import U, doubles, stored, types
from paper_2001_00138_amd import binding as B
from test_gpu_rms import TINY, chain, check_codes

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
# rows that share a wavefront, have one, several, with two and four runs a lane, and are read twice
COLS = [5, 100, 300, 513, 4096, 10000, 20000, 40000]


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def check(torch, rows, kind, eps, normal):
    """rows [n][cols] in `kind`, with ordinary ones beside them, keep their results; `normal`: those that do."""
    x = stored(torch, rows, kind)
    gamma = np.linspace(-1.5, 1.5, rows.shape[1]).astype(np.float32)
    y, s, rstd = ff.rms_norm(doubles(x), None, gamma, float(np.float32(eps)))
    rel = (chain(rows.shape[1]) / 2 + 8) * u
    args = dict(eps=eps, residual=torch.zeros_like(x).cuda())
    for out in ("f32", "bf16"):
        got, _, total, r = B.patdnn_rms_norm(x.cuda(), torch.from_numpy(gamma).cuda(), dtype=types(torch)[out], **args)
        assert (np.abs(doubles(r) - rstd) <= rel * rstd)[normal].all()
        assert (np.abs(doubles(got) - y) <= (rel + U[out] * (1 + rel)) * np.abs(y) + TINY[out])[normal].all()
        assert torch.equal(total.cpu(), x)
    codes, scales, _, _ = B.patdnn_rms_norm(x.cuda(), torch.from_numpy(gamma).cuda(), fp8=True, **args)
    check_codes(codes.cpu().numpy()[normal], scales.cpu().numpy()[normal], y[normal], rel * np.abs(y[normal]))
    return doubles(r)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_sum_of_squares_beyond_the_range(torch, cols, kind):
    """The sum of squares is 2^128 and more, the mean is not; where the mean is, too, rstd is 0."""
    rng = np.random.default_rng(cols)
    rows = rng.standard_normal((6, cols))
    for i, size in ((0, 1.2e19), (2, 1.8e19), (5, 1.1e19)):
        rows[i] = size * np.sign(rows[i])
    rows[3] = 3e38 * np.sign(rows[3])
    rows[4] *= 1e18
    assert (np.square(rows[[0, 2, 5]]).sum(axis=1) > 2.0 ** 128).all()
    rstd = check(torch, rows, kind, 1e-6, [0, 1, 2, 4, 5])
    assert rstd[3] == 0


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_squares_below_the_range(torch, cols, kind):
    """Squares that fp32 cannot hold, without an eps that they vanish beside; a larger value among them, and eps, come first where they are there."""
    rng = np.random.default_rng([cols, 1])
    rows = rng.standard_normal((7, cols))
    for i, size in ((0, 1e-19), (2, 1e-23), (3, 1e-30), (5, 3e-36)):
        rows[i] *= size
    rows[4] *= 1e-25
    rows[4, cols // 2] = 1e-3
    for eps in (0.0, 1e-42, 1e-31, 1e-6):
        check(torch, rows, kind, eps, slice(None))
