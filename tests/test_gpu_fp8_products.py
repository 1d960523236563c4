"""Products of fp8 codes on the GPU: linear layers, the gated pair of projections, its gradients, against the oracle.

Tolerance, u = 2^-24: products of codes and scales are exact; each of the K additions (and the joining of partial sums, fewer) rounds by at most u of what
it adds to, so K u of the sum of the terms' magnitudes.  Results in fewer bits than 32 come from the fp8 instruction, which adds groups of eight neighbouring
products and cuts each off at 2^-13 of the power of two of the largest: at most seven times that (the largest is whole).  SiLU's slope is at most 1.1, and its slope's at most 0.5; computing them
costs (|g| + 6) u of the value and (12 + 6 |g|) u; then half a spacing of the output's type."""

import numpy as np
import pytest

from oracle import feed_forward as ff
from oracle.operators import activation, activation_slope
from operator_helpers import U, doubles, guarded, replays, stored, types
from paper_2001_00138_amd import binding as B
from test_gpu_rms import TINY, check_codes

pytestmark = pytest.mark.gpu
KINDS = ["f32", "f16", "bf16"]
u = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def codes_of(torch, rng, rows, cols, squares=False):
    """Random values quantised by the oracle's rules (on the GPU, whose codes are tested beside this) -> (codes, scales, values)"""
    v = rng.standard_normal((rows, cols)) * np.exp(0.5 * rng.standard_normal((rows, 1)))
    codes, scales = B.patdnn_fp8_quantize(torch.from_numpy(v).float().cuda(), blocks="squares" if squares else "rows")
    return codes, scales, ff.fp8_values(codes.cpu().numpy(), scales.cpu().numpy(), cols)


def near(got, want, off, out):
    """Within `off` before the rounding to the output's type, which takes binary16 values of 65520 (half a spacing past the largest) and more to infinity."""
    with np.errstate(invalid="ignore"):
        fine = np.abs(got - want) <= off + U[out] * (np.abs(want) + off) + TINY[out]
    if out == "f16":
        fine |= np.isinf(got) & (np.sign(got) == np.sign(want)) & (np.abs(want) + off >= 65520)
    return fine.all()


def sums_of(x, w, out):
    z, size = x @ w.T, np.abs(x) @ np.abs(w).T
    off = x.shape[1] * u * size
    if out != "f32":
        pad = lambda t: np.abs(np.pad(t, ((0, 0), (0, -t.shape[1] % 8)))).reshape(t.shape[0], -1, 8)      # noqa: E731
        a, b = pad(x), pad(w)
        for g in range(a.shape[1]):
            off = off + 7 * 2.0 ** -13 * (a[:, None, g] * b[None, :, g]).max(axis=2)
    return z, off


def check_linear(torch, rows, k, n, squares, bias, act, out, pad=0):
    rng = np.random.default_rng([7, rows, k, n])
    xc, xs, x = codes_of(torch, rng, rows, k)
    wc, ws, w = codes_of(torch, rng, n, k, squares)
    b = rng.standard_normal(n).astype(np.float32) if bias else None
    z, off = sums_of(x, w, out)
    if bias:
        z = z + b
        off = off + u * np.abs(z)
    want = activation(z, act)
    off = 1.1 * off + (8 * u * np.abs(want) + u * np.abs(z * want) if act == "silu" else 0)
    to, check = guarded(torch, (rows, n + pad), types(torch)[out])
    B.patdnn_fp8_linear(xc, xs, wc, ws, None if b is None else torch.from_numpy(b).cuda(), to[:, :n], act=act)
    torch.cuda.synchronize()
    check()
    assert bool((to[:, n:] == 77).all())
    assert near(doubles(to[:, :n]), want, off, out)


def check_gated(torch, rows, k, n, squares, act, out, pad=0):
    rng = np.random.default_rng([8, rows, k, n])
    xc, xs, x = codes_of(torch, rng, rows, k)
    gc, gs, gate = codes_of(torch, rng, n, k, squares)
    uc, us, up = codes_of(torch, rng, n, k, squares)
    (g, eg), (v, ev) = sums_of(x, gate, out), sums_of(x, up, out)
    value = activation(g, act)
    want = value * v
    evalue = 1.1 * eg + (np.abs(g) + 6) * u * np.abs(value)
    off = evalue * (np.abs(v) + ev) + np.abs(value) * ev + 2 * u * np.abs(want)
    if out == "fp8":
        pieces = -(-n // 128)
        to, check = guarded(torch, (rows, pieces * 128), torch.uint8)
        scales, check2 = guarded(torch, (rows, pieces), torch.uint8)
        B.patdnn_fp8_gated(xc, xs, gc, gs, uc, us, to, scales=scales, act=act, fp8=True)
        torch.cuda.synchronize()
        check(), check2()
        check_codes(to.cpu().numpy(), scales.cpu().numpy(), want, off)
        return
    to, check = guarded(torch, (rows, n + pad), types(torch)[out])
    B.patdnn_fp8_gated(xc, xs, gc, gs, uc, us, to[:, :n], act=act)
    torch.cuda.synchronize()
    check()
    assert bool((to[:, n:] == 77).all())
    assert near(doubles(to[:, :n]), want, off, out)


def check_gated_backward(torch, rows, k, n, squares, act, out, dkind, pad=0):
    rng = np.random.default_rng([9, rows, k, n])
    xc, xs, x = codes_of(torch, rng, rows, k)
    gc, gs, gate = codes_of(torch, rng, n, k, squares)
    uc, us, up = codes_of(torch, rng, n, k, squares)
    dh = stored(torch, rng.standard_normal((rows, n)), dkind)
    (g, eg), (v, ev) = sums_of(x, gate, out), sums_of(x, up, out)
    value, slope, d = activation(g, act), activation_slope(g, act), np.abs(doubles(dh))
    dg, du = ff.gated_backward(doubles(dh), g, v, act)
    evalue = 1.1 * eg + (np.abs(g) + 6) * u * np.abs(value)
    eslope = 0.5 * eg + (12 + 6 * np.abs(g)) * u if act == "silu" else np.where(np.abs(g) <= eg, 1.0, 0.0) if act == "relu" else 0.0
    off = np.hstack((d * (ev * (np.abs(slope) + eslope) + np.abs(v) * eslope) + 2 * u * np.abs(dg), d * evalue + u * np.abs(du)))
    want = np.hstack((dg, du))
    to, check = guarded(torch, (rows, 2 * n + pad), types(torch)[out])
    on = torch.full((rows, n + pad), 5.0, dtype=dh.dtype, device="cuda")
    on[:, :n] = dh.cuda()
    B.patdnn_fp8_gated_backward(on[:, :n], xc, xs, gc, gs, uc, us, to[:, :2 * n], act=act)
    torch.cuda.synchronize()
    check()
    assert bool((to[:, 2 * n:] == 77).all())
    assert near(doubles(to[:, :2 * n]), want, off, out)


SIZES = [(1, 1, 1), (1, 128, 16), (2, 129, 17), (16, 300, 40), (17, 256, 128), (5, 1000, 130), (33, 511, 200), (64, 640, 64), (65, 385, 65), (1, 2100, 300),
         (130, 200, 257), (100, 1700, 300), (300, 130, 520)]


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("squares", [False, True])
def test_linear(torch, rows, k, n, squares):
    for i, out in enumerate(KINDS):
        check_linear(torch, rows, k, n, squares, bias=i != 1, act=["none", "relu", "silu"][(i + rows) % 3], out=out, pad=i * 3)


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("squares", [False, True])
def test_gated(torch, rows, k, n, squares):
    for i, out in enumerate(KINDS + ["fp8", "fp8"]):
        check_gated(torch, rows, k, n, squares, ["silu", "none", "relu"][(i + rows) % 3], out, pad=i * 3)


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("squares", [False, True])
def test_gated_backward(torch, rows, k, n, squares):
    for i, out in enumerate(KINDS):
        check_gated_backward(torch, rows, k, n, squares, ["silu", "none", "relu"][(i + rows) % 3], out, KINDS[(i + n) % 3], pad=i * 3)


@pytest.mark.parametrize("rows,k,n", [(1, 4096, 64), (16, 8192, 48), (40, 2048, 200), (200, 2048, 300)])
def test_whole_numbers_are_exact(torch, rows, k, n):
    """Whole numbers up to 15 and scales of one: sums below 2^24 have no rounding, in any order."""
    rng = np.random.default_rng([rows, k])
    x, w = rng.integers(-15, 16, (rows, k)).astype(np.float64), rng.integers(-15, 16, (n, k)).astype(np.float64)
    one = lambda v: (torch.from_numpy(v).float().to(torch.float8_e4m3fn).cuda(), torch.full((v.shape[0], k // 128), 127, dtype=torch.uint8, device="cuda"))      # noqa: E731
    got = B.patdnn_fp8_linear(*one(x), *one(w))
    assert (doubles(got) == x @ w.T).all()
    both = B.patdnn_fp8_gated_backward(torch.ones(rows, n, device="cuda"), *one(x), *one(w), *one(w[::-1].copy()), act="none")
    assert (doubles(both) == np.hstack((x @ w[::-1].T, x @ w.T))).all()


@pytest.mark.parametrize("rows", [1, 20, 150])
def test_scales_far_apart_and_not_finite(torch, rows):
    """Every row, and every piece of k, has a scale of its own; a block that is not finite makes its sums NaN and no others."""
    rng = np.random.default_rng(rows)
    k, n = 700, 150
    v, w = rng.standard_normal((rows, k)) * np.exp2(rng.integers(-20, 20, (rows, 1))), rng.standard_normal((n, k)) * np.exp2(rng.integers(-20, 20, (n, 1)))
    v *= np.exp2(np.repeat(rng.integers(-3, 3, 6), 128)[:k])
    xc, xs = B.patdnn_fp8_quantize(torch.from_numpy(v).float().cuda())
    w[7, 300] = np.nan
    wc, ws = B.patdnn_fp8_quantize(torch.from_numpy(w).float().cuda())
    got = doubles(B.patdnn_fp8_linear(xc, xs, wc, ws))
    assert np.isnan(got[:, 7]).all()
    keep = np.arange(n) != 7
    z, off = sums_of(ff.fp8_values(xc.cpu().numpy(), xs.cpu().numpy(), k), ff.fp8_values(wc.cpu().numpy(), ws.cpu().numpy(), k)[keep], "f32")
    assert (np.abs(got[:, keep] - z) <= off + u * np.abs(z)).all()
    xs[rows - 1, 2] = 255
    got = B.patdnn_fp8_gated(xc, xs, wc, ws, wc, ws, fp8=True)
    assert bool((got[1][rows - 1] == 255).all()) and bool((got[1][:rows - 1, 0] == 255).all()) and bool((got[1][:rows - 1, 1] != 255).all())


def test_graph_and_no_rows(torch):
    rng = np.random.default_rng(4)
    x = torch.randn(70, 400, device="cuda")
    gc, gs, _ = codes_of(torch, rng, 200, 400, True)
    uc, us, _ = codes_of(torch, rng, 200, 400, True)
    wc, ws, _ = codes_of(torch, rng, 400, 200, True)
    xc, xs = B.patdnn_fp8_quantize(x)
    h, hs = B.patdnn_fp8_gated(xc, xs, gc, gs, uc, us, fp8=True)
    out = B.patdnn_fp8_linear(h, hs, wc, ws)
    d = B.patdnn_fp8_gated_backward(x[:, :200], xc, xs, gc, gs, uc, us)
    rooms = [torch.empty(1 << 20, dtype=torch.uint8, device="cuda") for _ in range(3)]

    def call():
        B.patdnn_fp8_quantize(x, xc, xs)
        B.patdnn_fp8_gated(xc, xs, gc, gs, uc, us, h, scales=hs, fp8=True, workspace=rooms[0])
        B.patdnn_fp8_linear(h, hs, wc, ws, None, out, workspace=rooms[1])
        B.patdnn_fp8_gated_backward(x[:, :200], xc, xs, gc, gs, uc, us, d, workspace=rooms[2])
    for got, want in replays(torch, call, lambda: [xc, xs, h, hs, out, d], lambda i: x.normal_(0, 1 + i)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert B.patdnn_fp8_linear(xc[:0], xs[:0], gc, gs).shape == (0, 200)
    assert B.patdnn_fp8_gated(xc[:0], xs[:0], gc, gs, uc, us, fp8=True)[0].shape == (0, 256)
    assert B.patdnn_fp8_gated_backward(x[:0, :200], xc[:0], xs[:0], gc, gs, uc, us).shape == (0, 400)


# (sizes that take each tile shape, with rows and outputs that end inside a tile, and k of one to nine stages; and slices of k, of eight pieces and more, the last of
# three; and long sums in as few of the larger tiles as take them; and one to six stages where a CU has one tile of 128 by 128, of
# linear layers and of the gated pair; and slices of its tiles of 64 outputs by 128 rows)
LARGE = [(4090, 300, 4100), (2100, 520, 2000), (520, 1100, 700), (8200, 128, 2050), (300, 1030, 33000), (40, 5000, 300), (70, 4100, 1000), (20, 7200, 130),
         (3500, 6200, 3600), (1500, 6200, 2000), (300, 8200, 2000), (1500, 100, 2000), (2000, 250, 1590),
         (1030, 380, 3500), (2040, 500, 2040), (1900, 640, 1700), (1900, 700, 1700), (1800, 100, 1000), (1000, 370, 2000),
         (1000, 2100, 2000), (900, 8200, 700), (1400, 9000, 350)]


def whole(torch, rows, k, squares, seed):
    """Codes of whole numbers up to 15, scales 1/2, 1 and 2 -> (codes, scales, values)"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    pieces = -(-k // 128)
    v = torch.randint(-15, 16, (rows, pieces * 128), generator=g, device="cuda").float()
    v[:, k:] = 0
    scales = torch.randint(126, 129, (-(-rows // 128) if squares else rows, pieces), generator=g, device="cuda", dtype=torch.uint8)
    unit = torch.exp2(scales.double() - 127)
    if squares:
        unit = unit.repeat_interleave(128, dim=0)[:rows]
    return v.to(torch.float8_e4m3fn), scales, (v.double().view(rows, pieces, 128) * unit[:, :, None]).view(rows, -1)


@pytest.mark.parametrize("rows,k,n", LARGE)
@pytest.mark.parametrize("squares", [False, True])
def test_tiles_are_exact(torch, rows, k, n, squares):
    """Sums of whole numbers and quarters below 2^22 have no rounding: every tile shape equals the product in 64 bits."""
    (xc, xs, x), (gc, gs, gate), (uc, us, up) = whole(torch, rows, k, False, 1), whole(torch, n, k, squares, 2), whole(torch, n, k, squares, 3)
    g, v = x @ gate.t().contiguous(), x @ up.t().contiguous()
    for kind in KINDS:
        t = types(torch)[kind]
        out, check = guarded(torch, (rows, n + 3), t)
        B.patdnn_fp8_linear(xc, xs, gc, gs, None, out[:, :n])
        check()
        assert torch.equal(out[:, :n], g.float().to(t)) and bool((out[:, n:] == 77).all())
        out, check = guarded(torch, (rows, n + 3), t)
        B.patdnn_fp8_gated(xc, xs, gc, gs, uc, us, out[:, :n], act="relu")
        check()
        assert torch.equal(out[:, :n], (torch.relu(g).float() * v.float()).to(t)) and bool((out[:, n:] == 77).all())
        out, check = guarded(torch, (rows, 2 * n + 3), t)
        B.patdnn_fp8_gated_backward(torch.ones(rows, n, device="cuda", dtype=torch.bfloat16), xc, xs, gc, gs, uc, us, out[:, :2 * n], act="relu")
        check()
        want = torch.cat((torch.where(g > 0, v, 0.0), torch.relu(g)), dim=1).float().to(t)
        assert torch.equal(out[:, :2 * n], want) and bool((out[:, 2 * n:] == 77).all())
    h = torch.relu(g).float() * v.float()
    pieces = -(-n // 128)
    codes, check = guarded(torch, (rows, pieces * 128), torch.uint8)
    scales, check2 = guarded(torch, (rows, pieces), torch.uint8)
    B.patdnn_fp8_gated(xc, xs, gc, gs, uc, us, codes, scales=scales, act="relu", fp8=True)
    check(), check2()
    want = B.patdnn_fp8_quantize(h)
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
