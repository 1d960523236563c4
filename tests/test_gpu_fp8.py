"""fp8 codes on the GPU: equal to the oracle's in all four layouts, and read back exactly."""

import numpy as np
import pytest

from oracle import feed_forward as ff
from operator_helpers import doubles, guarded, replays, stored, types
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
    # ties and their neighbours, largest values at the border of a scale
    at = rng.random((rows, cols)) < 0.2
    ties = rng.choice([1.0625, 1.1875, 17 / 16, 464, 448, 450, 2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -10, 0.0, -0.0, 436, -436], (rows, cols))
    return np.where(at, ties * np.exp2(rng.integers(-3, 3, (rows, 1))), v)


def _check(torch, x, wide, squares, transposed):
    rows, cols = x.shape
    kind = {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[x.dtype]
    host = doubles(x).T if transposed else doubles(x)
    wc, ws = ff.fp8_quantize(host, squares)
    on = torch.full((rows, cols + wide), 9e9 if kind != "f16" else 6e4, dtype=x.dtype, device="cuda")
    on[:, :cols] = x.cuda()
    codes, check = guarded(torch, wc.shape, torch.uint8)
    scales, check2 = guarded(torch, ws.shape, torch.uint8)
    B.patdnn_fp8_quantize(on[:, :cols], codes, scales, blocks="squares" if squares else "rows", transposed=transposed)
    torch.cuda.synchronize()
    check()
    check2()
    assert (scales.cpu().numpy() == ws).all()
    assert (codes.cpu().numpy() == wc).all()
    for to in KINDS:
        out, check = guarded(torch, (host.shape[0], host.shape[1] + 3), types(torch)[to])
        B.patdnn_fp8_dequantize(codes, scales, host.shape[1], out[:, :host.shape[1]])
        torch.cuda.synchronize()
        check()
        want = torch.from_numpy(ff.fp8_values(wc, ws, host.shape[1])).to(types(torch)[to])
        got = out[:, :host.shape[1]].cpu()
        assert bool((out[:, host.shape[1]:] == 77).all())
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0, 1, -1), want.nan_to_num(0, 1, -1))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (2, 129), (7, 500), (128, 128), (127, 130), (129, 127), (300, 24), (3, 2177), (257, 384)])
def test_quantise(torch, rows, cols, kind):
    x = stored(torch, _values(np.random.default_rng([12, rows, cols]), rows, cols), kind)
    for squares in (False, True):
        for transposed in (False, True):
            _check(torch, x, 0 if rows % 2 else 5, squares, transposed)


@pytest.mark.parametrize("kind", KINDS)
def test_extremes(torch, kind):
    top = torch.finfo(types(torch)[kind])
    tiny = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}[kind]
    x = torch.zeros(12, 200, dtype=types(torch)[kind])
    x[0, 0], x[0, 1] = top.max, top.min
    x[1, 5], x[1, 6] = tiny, -3 * tiny
    x[2, :] = top.tiny
    x[3, 3] = float("inf")
    x[4, 140] = float("-inf")
    x[5, 127], x[5, 128] = float("nan"), 1.0
    x[6, :128] = top.min                                    # masks of the type's lowest value
    x[7, 0], x[7, 1:128] = 1e4, 1e-4
    x[8, :] = -0.0
    x[9, 0], x[9, 1] = float("nan"), float("inf")
    x[10, :] = torch.linspace(-448, 448, 200)
    for squares in (False, True):
        for transposed in (False, True):
            _check(torch, x, 1, squares, transposed)


def test_all_codes_and_scales(torch):
    """Every scale with every code, read back to all types: the value rounded once."""
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1).contiguous()
    scales = torch.arange(256, dtype=torch.uint8).view(256, 1).repeat(1, 2).contiguous()
    want = torch.from_numpy(ff.fp8_values(codes.numpy(), scales.numpy(), 256))
    for kind in KINDS:
        got = B.patdnn_fp8_dequantize(codes.cuda(), scales.cuda(), 256, dtype=types(torch)[kind]).cpu()
        w = want.to(torch.float32).to(types(torch)[kind])    # (four bits: the first rounding is exact down to 2^-149)
        assert torch.equal(got.isnan(), w.isnan()) and torch.equal(got.nan_to_num(0, 1, -1), w.nan_to_num(0, 1, -1))
    as_torch = B.patdnn_fp8_dequantize(codes.cuda().view(torch.float8_e4m3fn), scales.cuda().view(torch.float8_e8m0fnu), 256)
    assert torch.equal(as_torch.cpu().nan_to_num(0, 1, -1), want.float().nan_to_num(0, 1, -1))


def test_far_rows(torch):
    """Rows whose offsets pass 2^31 elements: the same rows, near."""
    row = (1 << 31) // 3 + 5
    x = torch.empty(4 * row, dtype=torch.bfloat16, device="cuda").as_strided((4, 300), (row, 1))
    x.copy_(torch.randn(4, 300, device="cuda"))
    for squares in ("rows", "squares"):
        for transposed in (False, True):
            far = B.patdnn_fp8_quantize(x, blocks=squares, transposed=transposed)
            near = B.patdnn_fp8_quantize(x.contiguous(), blocks=squares, transposed=transposed)
            assert all(torch.equal(a, b) for a, b in zip(far, near))


def test_graph_and_no_rows(torch):
    x = torch.randn(200, 333, device="cuda", dtype=torch.float16)
    codes, scales = B.patdnn_fp8_quantize(x, transposed=True)
    out = B.patdnn_fp8_dequantize(codes, scales, 200)

    def call():
        B.patdnn_fp8_quantize(x, codes, scales, transposed=True)
        B.patdnn_fp8_dequantize(codes, scales, 200, out)
    for got, want in replays(torch, call, lambda: [codes, scales, out], lambda i: x.normal_(0, 1 + i)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    c, s = B.patdnn_fp8_quantize(x[:0])
    assert c.shape == (0, 384) and B.patdnn_fp8_dequantize(c, s, 333).shape == (0, 333)
    assert B.patdnn_fp8_quantize(x[:0], transposed=True)[0].shape == (333, 0)
