"""MXFP4 on the GPU: codes and scales equal to the oracle's, linear layers within the rounding of their sums.

Tolerance of a linear layer: products of codes and scales are exact, each of the K additions (and the joining of partial
sums, fewer) rounds by at most 2^-24 of what it adds to, so K 2^-24 of the sum of the terms' magnitudes; an activation's slope is
at most 1.1 and SiLU's own operations round by a few 2^-24 times |z|; then half a spacing of the output's type."""

import numpy as np
import pytest

from oracle import operators as oo
from operator_helpers import U, doubles, guarded, replays, stored, types
from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu
KINDS = ["f32", "f16", "bf16"]


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _values(rng, rows, cols):
    v = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))
    # ties and their neighbours, at scales of their own
    at = rng.random((rows, cols)) < 0.3
    ties = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 0.0, -0.0, -2.5, -0.25], (rows, cols))
    return np.where(at, ties * np.exp2(rng.integers(-3, 3, (rows, 1))), v)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (2, 32), (3, 33), (5, 127), (4, 128), (3, 129), (7, 500), (2, 2048), (1, 2177), (40, 64), (300, 24)])
def test_quantise(torch, rows, cols, kind):
    rng = np.random.default_rng([11, rows, cols])
    x = stored(torch, _values(rng, rows, cols), kind)
    pieces = -(-cols // 128)
    codes, check = guarded(torch, (rows, pieces * 64), torch.uint8, fill=77)
    scales, check2 = guarded(torch, (rows, pieces * 4), torch.uint8, fill=77)
    B.patdnn_mxfp4_quantize(x.cuda(), codes, scales)
    torch.cuda.synchronize()
    check()
    check2()
    wc, ws = oo.mxfp4_quantize(doubles(x))
    assert (scales.cpu().numpy() == ws).all() and (codes.cpu().numpy() == wc).all()
    out, check = guarded(torch, (rows, cols), types(torch)[kind])
    B.patdnn_mxfp4_dequantize(codes, scales, cols, out)
    torch.cuda.synchronize()
    check()
    want = torch.from_numpy(oo.mxfp4_values(wc, ws, cols)).to(types(torch)[kind])
    assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("kind", KINDS)
def test_extremes(torch, kind):
    top = torch.finfo(types(torch)[kind])
    tiny = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}[kind]
    x = torch.zeros(12, 64, dtype=types(torch)[kind])
    x[0, 0], x[0, 1] = top.max, top.min
    x[1, 5], x[1, 6] = tiny, -3 * tiny
    x[2, :] = top.tiny
    x[3, 3] = float("inf")
    x[4, 40] = float("-inf")
    x[5, 31], x[5, 32] = float("nan"), 1.0
    x[6, :32] = top.min                                     # masks of the type's lowest value
    x[7, 0], x[7, 1:32] = 1e4, 1e-4
    x[8, :] = -0.0
    x[9, 0] = float("nan")
    x[9, 1] = float("inf")
    x[10, :] = torch.linspace(-8, 8, 64)
    codes, scales = B.patdnn_mxfp4_quantize(x.cuda())
    wc, ws = oo.mxfp4_quantize(doubles(x))
    assert (scales.cpu().numpy() == ws).all() and (codes.cpu().numpy() == wc).all()
    for other in KINDS:
        got = B.patdnn_mxfp4_dequantize(codes, scales, 64, dtype=types(torch)[other]).cpu()
        want = torch.from_numpy(oo.mxfp4_values(wc, ws, 64)).float().to(types(torch)[other])
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


def test_all_codes_and_scales(torch):
    codes = torch.arange(256, dtype=torch.uint8).repeat_interleave(64).view(256, 64).clone()
    codes[:, 1::2] = torch.arange(256, dtype=torch.uint8).flip(0)[:, None]
    scales = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 4)
    want = oo.mxfp4_values(codes.numpy(), scales.numpy(), 128).astype(np.float32)
    got = B.patdnn_mxfp4_dequantize(codes.cuda(), scales.cuda(), 128).cpu().numpy()
    assert (np.isnan(got) == np.isnan(want)).all() and (np.nan_to_num(got, nan=0) == np.nan_to_num(want, nan=0)).all()


@pytest.mark.parametrize("wide,offset", [(200, 0), (205, 3), (216, 16)])
def test_rows_of_wider_tensors(torch, wide, offset):
    x = torch.randn(9, wide, device="cuda").half()
    part = x[:, offset:offset + 150]
    a, b = B.patdnn_mxfp4_quantize(part), B.patdnn_mxfp4_quantize(part.contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    whole = torch.full((9, wide), 3.0, device="cuda")
    B.patdnn_mxfp4_dequantize(*a, 150, whole[:, offset:offset + 150])
    assert torch.equal(whole[:, offset:offset + 150], B.patdnn_mxfp4_dequantize(*a, 150))
    assert bool((whole[:, :offset] == 3).all()) and bool((whole[:, offset + 150:] == 3).all())
    # one row for all
    one = x[:1, :150].expand(9, 150)
    assert torch.equal(B.patdnn_mxfp4_quantize(one)[0], B.patdnn_mxfp4_quantize(one.contiguous())[0])


def _linear(torch, rows, k, out, kind, dst, act, quantised=False, bias=True, seed=1, x_wide=0, out_wide=0):
    rng = np.random.default_rng([seed, rows, k, out])
    x = stored(torch, rng.standard_normal((rows, k)) * np.exp(0.5 * rng.standard_normal((rows, 1))), kind)
    w = rng.standard_normal((out, k)).astype(np.float32) * np.float32(np.sqrt(2 / k))
    b = rng.standard_normal(out).astype(np.float32) if bias else None
    wc, ws = B.patdnn_mxfp4_quantize(torch.from_numpy(w).cuda())
    xc, xs = (t.cpu().numpy() for t in B.patdnn_mxfp4_quantize(x.cuda()))
    xv = oo.mxfp4_values(xc, xs, k)
    want, size = oo.linear(xv, oo.mxfp4_values(wc.cpu().numpy(), ws.cpu().numpy(), k), b, act)
    whole, check = guarded(torch, (rows, out + out_wide), types(torch)[dst])
    whole.fill_(31)
    xt = x.cuda()
    if x_wide:
        wider = torch.full((rows, k + x_wide), float("nan"), dtype=xt.dtype, device="cuda")
        wider[:, :k] = xt
        xt = wider[:, :k]
    more = {"x_scales": torch.from_numpy(xs).cuda()} if quantised else {}
    got = B.patdnn_mxfp4_linear(torch.from_numpy(xc).cuda() if quantised else xt, wc, ws, None if b is None else torch.from_numpy(b).cuda(),
                                whole[:, :out], act=act, **more)
    torch.cuda.synchronize()
    check()
    assert bool((whole[:, out:] == 31).all())
    allowed = 1.1 * (k + 2) * U["f32"] * size + (8 * U["f32"] * (1 + size) * np.abs(want) if act == "silu" else 0) + \
        (U[dst] * np.abs(want) * 1.01 + 2.0 ** -24 if dst != "f32" else 0)
    worst = (np.abs(doubles(got) - want) - allowed).max()
    assert worst <= 0, worst


# rows of one and few, tiles of 16, 64, 128 and 256 rows and outputs and their neighbours, pieces of 128 along k and their neighbours
@pytest.mark.parametrize("rows", [1, 2, 5, 15, 16, 17, 31, 33, 64, 77, 128, 129, 200, 257, 300])
@pytest.mark.parametrize("k,out", [(1, 1), (127, 17), (128, 16), (300, 70), (515, 129), (1024, 260), (2100, 96)])
def test_linear_sizes(torch, rows, k, out):
    kinds = KINDS[(rows + k) % 3], KINDS[(rows + out) % 3]
    _linear(torch, rows, k, out, *kinds, ["none", "relu", "silu"][(rows + k + out) % 3], quantised=(rows + out) % 2 == 1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dst", KINDS)
@pytest.mark.parametrize("rows", [3, 100])
def test_linear_types(torch, rows, kind, dst):
    for act in ("none", "relu", "silu"):
        _linear(torch, rows, 200, 50, kind, dst, act)
        _linear(torch, rows, 200, 50, kind, dst, act, bias=False, x_wide=5, out_wide=3)
        _linear(torch, rows, 256, 64, kind, dst, act, quantised=True, out_wide=64, x_wide=0)


@pytest.mark.parametrize("rows,k,out", [(1, 25088, 300), (9, 12000, 1000), (70, 9000, 40), (1000, 700, 600), (2500, 128, 512), (600, 2000, 1030)])
def test_linear_larger(torch, rows, k, out):
    _linear(torch, rows, k, out, "f16", "f32", "none")
    _linear(torch, rows, k, out, "bf16", "bf16", "relu", quantised=True)


# few rows on either side of each choice: in one launch or two, by rows or in tiles, with one and more tiles of rows
@pytest.mark.parametrize("rows,k,out", [(4, 12900, 33), (4, 12700, 33), (5, 300, 4200), (20, 300, 4112), (63, 500, 4400), (20, 1500, 2100), (20, 2100, 2100), (13, 5000, 900),
                                        (12, 4100, 900), (48, 4100, 700), (37, 4200, 1400), (63, 8192, 70), (63, 8193, 70), (17, 8300, 70)])
def test_linear_few_rows(torch, rows, k, out):
    _linear(torch, rows, k, out, "f16", "f32", "silu")
    _linear(torch, rows, k, out, "f32", "f16", "none", quantised=True)


# more outputs or rows than a workgroup a CU takes: tiles, of every size and with their ends inside
@pytest.mark.parametrize("rows", [5, 17, 64, 77, 130, 300, 1025])
@pytest.mark.parametrize("k,out", [(1, 4400), (515, 4099), (1300, 4112), (2100, 4353), (2600, 1030), (8200, 270)])
def test_linear_many_outputs(torch, rows, k, out):
    kinds = KINDS[(rows + k) % 3], KINDS[(rows + out) % 3]
    _linear(torch, rows, k, out, *kinds, ["none", "relu", "silu"][(rows + k + out) % 3], quantised=True)
    if (rows + out) % 2:
        _linear(torch, rows, k, out, *kinds, "relu", out_wide=3, x_wide=5)


@pytest.mark.parametrize("rows", [2, 40, 300])
def test_linear_is_exact_where_sums_are(torch, rows):
    """Small whole numbers: every sum is exact, whatever its order, so outputs are equal."""
    rng = np.random.default_rng(12)
    x = rng.integers(-3, 4, (rows, 700)).astype(np.float32)
    w = rng.integers(-3, 4, (333, 700)).astype(np.float32)
    x[:, ::32], w[:, ::32] = 4, 4                              # units of 1 in every block
    got = B.patdnn_mxfp4_linear(torch.from_numpy(x).cuda(), *B.patdnn_mxfp4_quantize(torch.from_numpy(w).cuda()))
    assert (got.cpu().numpy() == x @ w.T).all()


@pytest.mark.parametrize("rows", [1, 20, 200])
def test_linear_not_finite(torch, rows):
    """What is not finite in a row of x reaches that row's outputs, in a row of the weights that output's, and nothing else."""
    x, w = torch.randn(rows, 300, device="cuda"), torch.randn(90, 300, device="cuda")
    codes = B.patdnn_mxfp4_quantize(w)
    want = B.patdnn_mxfp4_linear(x, *codes)
    x[rows // 2, 299] = float("inf")
    w[17, 5] = float("nan")
    got = B.patdnn_mxfp4_linear(x, *B.patdnn_mxfp4_quantize(w), act="relu")
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[rows // 2] = True
    hit[:, 17] = True
    assert bool(got[hit].isnan().all()) and torch.equal(got[~hit], want.relu()[~hit])


def test_linear_repeats_and_ignores_the_workspace(torch):
    x, w = torch.randn(130, 3000, device="cuda").half(), torch.randn(77, 3000, device="cuda")
    codes = B.patdnn_mxfp4_quantize(w)
    a = B.patdnn_mxfp4_linear(x, *codes)
    needs = B.patdnn_mxfp4_linear_workspace_bytes(130, 3000, 77, x_type=B.PATDNN_F16, out_type=B.PATDNN_F16)
    for fill in (0, 255):
        work = torch.full((needs + 100,), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(a, B.patdnn_mxfp4_linear(x, *codes, workspace=work)) and bool((work[needs:] == fill).all())
    with pytest.raises(B.PatdnnError) as e:
        B.patdnn_mxfp4_linear(x, *codes, workspace=torch.empty(max(0, needs - 1), dtype=torch.uint8, device="cuda"))
    assert e.value.status == B.PATDNN_EINVAL


def test_no_rows(torch):
    x = torch.empty(0, 200, device="cuda")
    codes, scales = B.patdnn_mxfp4_quantize(x)
    assert codes.shape == (0, 128) and B.patdnn_mxfp4_dequantize(codes, scales, 200).shape == (0, 200)
    w = B.patdnn_mxfp4_quantize(torch.randn(7, 200, device="cuda"))
    assert B.patdnn_mxfp4_linear(x, *w).shape == (0, 7)


def test_offsets_beyond_32_bits(torch):
    rows, k, out = 20, 256, 48
    whole = torch.zeros((1 << 32) + 65536, dtype=torch.int8, device="cuda").view(torch.bfloat16)
    stride = (whole.numel() - 512) // (rows - 1) // 8 * 8
    x = torch.randn(rows, k, device="cuda").bfloat16()
    far = torch.as_strided(whole, (rows, k), (stride, 1))
    far.copy_(x)
    w = B.patdnn_mxfp4_quantize(torch.randn(out, k, device="cuda"))
    a, b = B.patdnn_mxfp4_quantize(far), B.patdnn_mxfp4_quantize(x)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for m in (3, rows):                                         # in one launch, and quantised before
        want = B.patdnn_mxfp4_linear(x[:m], *w)
        assert torch.equal(B.patdnn_mxfp4_linear(far[-m:], *w), B.patdnn_mxfp4_linear(x[-m:].contiguous(), *w))
        far.zero_()
        B.patdnn_mxfp4_linear(x[:m], *w, out=far[rows - m:, :out])
        assert torch.equal(far[rows - m:, :out], want)
        far.copy_(x)
    B.patdnn_mxfp4_dequantize(*b, k, far)
    assert torch.equal(far, B.patdnn_mxfp4_dequantize(*b, k, dtype=torch.bfloat16))


@pytest.mark.parametrize("rows", [2, 70])
def test_streams_and_graphs(torch, rows):
    x = torch.randn(rows, 400, device="cuda")
    w = B.patdnn_mxfp4_quantize(torch.randn(50, 400, device="cuda"))
    codes, scales = B.patdnn_mxfp4_quantize(x)
    values, out = torch.empty_like(x), torch.empty(rows, 50, device="cuda")
    work = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def call():
        B.patdnn_mxfp4_quantize(x, codes, scales)
        B.patdnn_mxfp4_dequantize(codes, scales, 400, values)
        B.patdnn_mxfp4_linear(x, *w, out=out, workspace=work)
    for got, want in replays(torch, call, lambda: [codes, scales, values, out], lambda i: x.normal_()):
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        got = B.patdnn_mxfp4_linear(x, *w, stream=stream)
        side.synchronize()
        assert torch.equal(got, out)
