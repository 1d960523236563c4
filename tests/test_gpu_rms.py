"""Root-mean-square norm on the GPU against the oracle.

Tolerances, u = 2^-24: the sum of squares is positive terms added in chains (eight values a run, up to four runs a lane or
more where rows are read twice, six steps over lanes, sixteen wavefronts): CHAIN u relative, so half of that on rstd; s, its square, the mean, the root
and the products are a rounding each.  A result is then off by (CHAIN / 2 + 8) u of itself and half a spacing of its type.  Backward, the sum
of d xh is off by (CHAIN + 4) u of the sum of its terms' magnitudes."""

import numpy as np
import pytest

from oracle import feed_forward as ff
from operator_helpers import U, doubles, guarded, replays, stored, types
from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu
KINDS = ["f32", "f16", "bf16"]
u = 2.0 ** -24
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}      # half the spacing of subnormal results


def chain(cols):
    return 8 * max(4, -(-cols // 8192)) + 6 + 16


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _inputs(torch, rows, cols, kind, seed=0, wide=0):
    rng = np.random.default_rng([seed, rows, cols])
    spread = np.exp(0.5 * rng.standard_normal(cols))
    x, res = (stored(torch, rng.standard_normal((rows, cols)) * spread * k, kind) for k in (1, 2))
    gamma = (1 + 0.3 * rng.standard_normal(cols)).astype(np.float32)

    def place(t):
        on = torch.full((rows, cols + wide), 55.0, dtype=t.dtype, device="cuda")
        on[:, :cols] = t.cuda()
        return on[:, :cols]
    return rng, x, res, gamma, place


def check_codes(codes, scales, y, off):
    """Codes of y known to within `off`: the scale of a largest magnitude in reach, then every value at most half a code away."""
    rows, cols = y.shape
    pieces = -(-cols // 128)
    v = np.zeros((rows, pieces * 128))
    v[:, :cols] = np.abs(y)
    o = np.zeros_like(v)
    o[:, :cols] = off
    fine = lambda top: np.where(top > 0, np.maximum(-127, np.ceil(np.log2(np.maximum(top, 1e-300) / 448))), -127) + 127      # noqa: E731
    low = fine((v - o).reshape(rows, pieces, 128).max(axis=2) * (1 - 1e-14))
    high = fine((v + o).reshape(rows, pieces, 128).max(axis=2) * (1 + 1e-14))
    assert ((scales >= low) & (scales <= high)).all()
    unit = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 128, axis=1)[:, :cols]
    got = ff.fp8_values(codes, scales, cols)
    assert (np.abs(got - y) <= np.maximum(2.0 ** -4 * (np.abs(y) + off), 2.0 ** -10 * unit) + off).all()
    assert not codes[:, cols:].any()


SIZES = [(1, 1), (3, 5), (20, 64), (17, 128), (9, 130), (5, 256), (2, 300), (7, 511), (6, 513), (3, 1000), (2, 4096), (3, 4100), (2, 5120), (1, 8192), (2, 8200),
         (2, 16384), (1, 20000), (1, 33000), (1, 1 << 20), (300, 40)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(torch, rows, cols, kind):
    wide = 3 if cols % 2 else 0
    rng, x, res, gamma, place = _inputs(torch, rows, cols, kind, wide=wide)
    for residual in (False, True):
        y, s, rstd = ff.rms_norm(doubles(x), doubles(res) if residual else None, gamma, 1e-6)
        rel = (chain(cols) / 2 + 8) * u
        for out in KINDS + ["fp8"]:
            total, check = guarded(torch, (rows, cols + wide), types(torch)[kind])
            r, check2 = guarded(torch, (rows,), torch.float32)
            args = dict(residual=place(res) if residual else None, sum=total[:, :cols], rstd=r, fp8=out == "fp8")
            if out == "fp8":
                pieces = -(-cols // 128)
                to, check3 = guarded(torch, (rows, pieces * 128), torch.uint8)
                scales, check4 = guarded(torch, (rows, pieces), torch.uint8)
                B.patdnn_rms_norm(place(x), torch.from_numpy(gamma).cuda(), to, scales=scales, **args)
                torch.cuda.synchronize()
                check4()
                check_codes(to.cpu().numpy(), scales.cpu().numpy(), y, rel * np.abs(y))
            else:
                to, check3 = guarded(torch, (rows, cols + wide), types(torch)[out])
                B.patdnn_rms_norm(place(x), torch.from_numpy(gamma).cuda(), to[:, :cols], **args)
                torch.cuda.synchronize()
                assert (np.abs(doubles(to[:, :cols]) - y) <= (rel + U[out] * (1 + rel)) * np.abs(y) + TINY[out]).all()
                assert bool((to[:, cols:] == 77).all())
            check(), check2(), check3()
            assert (np.abs(doubles(total[:, :cols]) - s) <= (U[kind] + 2 * u) * np.abs(s) + TINY[kind]).all() and bool((total[:, cols:] == 77).all())
            assert (np.abs(doubles(r) - rstd) <= rel * rstd).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [*SIZES, (1300, 100), (600, 1030), (700, 520)])
def test_backward(torch, rows, cols, kind):
    wide = 3 if cols % 2 else 0
    rng, s, _, gamma, place = _inputs(torch, rows, cols, kind, seed=1, wide=wide)
    r = (1 / np.sqrt((doubles(s) ** 2).mean(axis=1) + 1e-6)).astype(np.float32)
    for dkind, with_dsum, with_gamma in ((kind, True, True), ("f32", False, True), ("bf16", True, False), ("f16", False, False)):
        dy, dsum = stored(torch, rng.standard_normal((rows, cols)), dkind), stored(torch, rng.standard_normal((rows, cols)), kind)
        g = gamma if with_gamma else None
        dx, dgamma = ff.rms_norm_backward(doubles(dy), doubles(s), r, g, doubles(dsum) if with_dsum else None)
        out, check = guarded(torch, (rows, cols + wide), types(torch)[kind])
        dg, check2 = guarded(torch, (cols,), torch.float32)
        B.patdnn_rms_norm_backward(place(dy), place(s), torch.from_numpy(r).cuda(), None if g is None else torch.from_numpy(g).cuda(), out[:, :cols],
                                   dsum=place(dsum) if with_dsum else None, dgamma=dg)
        torch.cuda.synchronize()
        check(), check2()
        xh = np.abs(doubles(s) * r[:, None].astype(np.float64))
        d = np.abs(doubles(dy) * (1.0 if g is None else g.astype(np.float64)))
        mean = (d * xh).mean(axis=1, keepdims=True)
        rr = r[:, None].astype(np.float64)
        add = np.abs(doubles(dsum)) if with_dsum else 0.0
        off = u * (4 * rr * d + rr * xh * mean * (2 * chain(cols) + 12) + 2 * add)
        assert (np.abs(doubles(out[:, :cols]) - dx) <= off + U[kind] * (np.abs(dx) + off) + TINY[kind]).all()
        assert bool((out[:, cols:] == 77).all())
        size = (np.abs(doubles(dy)) * xh).sum(axis=0)
        # a workgroup's rows (two or three here), those that share it, and the joining of up to 650 workgroups by 32 half wavefronts: fewer than 64; 64 slabs where rows are
        # not held
        steps = max(rows // 512, rows // 64 if cols > 16384 else 0) + 16 + 32 + 16
        assert (np.abs(doubles(dg) - dgamma) <= (steps + 3) * u * size + 2.0 ** -149).all()


@pytest.mark.parametrize("rows,cols", [(3, 200), (2, 3000), (2, 40000)])
def test_in_place(torch, rows, cols):
    """sum=residual, and the gradient into dsum, give the bits of the calls apart."""
    torch.manual_seed(rows)
    x, res, dy, dsum = (torch.randn(rows, cols, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    y, _, s, rstd = B.patdnn_rms_norm(x, residual=res)
    kept = res.clone()
    y2, _, s2, rstd2 = B.patdnn_rms_norm(x, residual=kept, sum=kept)
    assert s2 is kept and torch.equal(y, y2) and torch.equal(s, s2) and torch.equal(rstd, rstd2)
    dx, dg = B.patdnn_rms_norm_backward(dy, s, rstd, dsum=dsum)
    kept = dsum.clone()
    dx2, dg2 = B.patdnn_rms_norm_backward(dy, s, rstd, dsum=kept, out=kept)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2)


@pytest.mark.parametrize("cols", [100, 3000, 40000])
def test_not_finite_stays_in_its_row(torch, cols):
    torch.manual_seed(cols)
    x = torch.randn(5, cols, device="cuda")
    bad = x.clone()
    bad[1, 7], bad[3, cols - 1] = float("nan"), float("inf")
    bad[2] = 0
    y, _, _, rstd = B.patdnn_rms_norm(bad, eps=0.0)
    good, _, _, _ = B.patdnn_rms_norm(x, eps=0.0)
    assert torch.equal(y[[0, 4]], good[[0, 4]]) and bool(y[1].isnan().all()) and bool(y[2].isnan().all())      # 0 times 1 / 0
    assert float(rstd[3]) == 0 and bool(y[3, -1].isnan()) and bool((y[3, :-1] == 0).all())
    codes, scales, _, _ = B.patdnn_rms_norm(bad, eps=0.0, fp8=True)
    assert bool((scales[1] == 255).all()) and int(scales[3, -1]) == 255 and int((scales[[0, 4]] == 255).sum()) == 0
    low = torch.full((2, cols), torch.finfo(torch.bfloat16).min, device="cuda", dtype=torch.bfloat16)      # squares beyond fp32
    assert bool((B.patdnn_rms_norm(low)[0] == 0).all())
    zero, _, _, r = B.patdnn_rms_norm(torch.zeros(2, cols, device="cuda"), eps=1e-6)
    assert bool((zero == 0).all()) and torch.allclose(r, torch.full_like(r, 1e3), rtol=1e-6)


def test_broadcast_gradient_far_rows_and_repeats(torch):
    torch.manual_seed(9)
    s = torch.randn(700, 300, device="cuda")
    rstd = torch.rsqrt(s.square().mean(dim=1) + 1e-6)
    dy = torch.randn(300, device="cuda").expand(700, 300)           # rows that lie on one another
    a, b = B.patdnn_rms_norm_backward(dy, s, rstd)
    c, d = B.patdnn_rms_norm_backward(dy.contiguous(), s, rstd)
    assert torch.equal(a, c) and torch.equal(b, d)
    row = (1 << 31) // 3 + 5
    far = torch.empty(4 * row, dtype=torch.bfloat16, device="cuda").as_strided((4, 300), (row, 1))
    far.copy_(torch.randn(4, 300, device="cuda"))
    near = far.contiguous()
    assert torch.equal(B.patdnn_rms_norm(far)[0], B.patdnn_rms_norm(near)[0])
    g = torch.randn(4, 300, device="cuda", dtype=torch.bfloat16)
    r = B.patdnn_rms_norm(near)[3]
    assert all(torch.equal(p, q) for p, q in zip(B.patdnn_rms_norm_backward(g, far, r), B.patdnn_rms_norm_backward(g, near, r)))
    y = far.new_empty(0)
    out = torch.empty(4 * row, dtype=torch.bfloat16, device="cuda").as_strided((4, 300), (row, 1))
    B.patdnn_rms_norm(near, out=out)
    assert torch.equal(out, B.patdnn_rms_norm(near)[0]) and y.numel() == 0


def test_no_rows(torch):
    x = torch.randn(0, 50, device="cuda")
    assert B.patdnn_rms_norm(x)[0].shape == (0, 50) and B.patdnn_rms_norm(x, fp8=True)[0].shape == (0, 128)
    dx, dgamma = B.patdnn_rms_norm_backward(x, x, torch.empty(0, device="cuda"), dgamma=torch.full((50,), 3.0, device="cuda"))
    assert dx.shape == (0, 50) and bool((dgamma == 0).all())


def test_graph(torch):
    x, res, dy = (torch.randn(40, 1500, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    gamma = torch.rand(1500, device="cuda")
    codes, scales, s, rstd = B.patdnn_rms_norm(x, gamma, residual=res, fp8=True)
    dx, dgamma = B.patdnn_rms_norm_backward(dy, s, rstd, gamma)
    room = torch.empty(64 * 1500, device="cuda")

    def call():
        B.patdnn_rms_norm(x, gamma, codes, residual=res, sum=s, scales=scales, rstd=rstd, fp8=True)
        B.patdnn_rms_norm_backward(dy, s, rstd, gamma, dx, dgamma=dgamma, workspace=room)
    for got, want in replays(torch, call, lambda: [codes, scales, s, rstd, dx, dgamma], lambda i: x.normal_(0, 1 + i)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
