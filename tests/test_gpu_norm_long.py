"""Group norm of as many pixels as it takes, one channel of them, against sums in 64 bits.

Tolerances: 128 slabs of 256 lanes leave each lane some 65536 values.  Rounding errors add up like a random walk: a lane's sum of squares, relative, by
sqrt(65536) 2^-24, and four times that is allowed for rstd; a sum of gradients by sqrt(M) 2^-24 times the largest partial sum of a lane, six
deviations, 6 sqrt(65536).  What is left out of the sums, one lane's values, would be 256 and more."""

import pytest

from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu
STEP = 1 << 27


def test_one_channel_of_two_billion_pixels():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    count = 2 ** 31 - 1025
    g = torch.Generator(device="cuda").manual_seed(6)
    x, dy = (torch.empty(1, count, 1, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, dy):
        for part in t.view(-1).split(STEP):
            part.normal_(generator=g)
    parts = lambda *tensors: zip(*(t.view(-1).split(STEP) for t in tensors))       # noqa: E731
    total = lambda f, *tensors: sum(f(*(p.double() for p in part)).sum().item() for part in parts(*tensors))   # noqa: E731
    mean = total(lambda a: a, x) / count
    rstd = (total(lambda a: (a - mean) ** 2, x) / count + 1e-5) ** -0.5
    gamma, beta = torch.tensor([1.5], device="cuda"), torch.tensor([-0.25], device="cuda")
    y, m, r = B.patdnn_group_norm(x, 1, gamma, beta)
    rough = 4 * 256 * 2.0 ** -24
    assert abs(m.item() - mean) <= 1e-6 and abs(r.item() - rstd) <= rough * rstd
    for a, b in parts(x, y):
        want = (a.double() - mean) * rstd * 1.5 - 0.25
        assert bool(((b.double() - want).abs() <= (2.0 ** -8 * 1.01 + rough) * want.abs() + rough).all())
    del y
    dx, dgamma, dbeta = B.patdnn_group_norm_backward(dy, x, m, r, 1, gamma, beta)
    mean, rstd = m.double().item(), r.double().item()
    a, b = total(lambda d: d, dy), total(lambda d, v: d * (v - mean) * rstd, dy, x)
    allowed = count ** 0.5 * 2.0 ** -24 * 6 * 256
    assert abs(dbeta.item() - a) <= allowed and abs(dgamma.item() - b) <= allowed
    for v, d, got in parts(x, dy, dx):
        want = rstd * 1.5 * (d.double() - a / count - (v.double() - mean) * rstd * (b / count))
        assert bool(((got.double() - want).abs() <= 2.0 ** -8 * 1.01 * want.abs() + 1e-6 * (1 + d.double().abs())).all())
