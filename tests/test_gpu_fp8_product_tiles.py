"""What the tile shapes of the products of fp8 codes make of their sums: bias, activations, and gradients from dh of every type, all elements of it different.

Sums are of whole numbers times a power of two, without rounding, so what follows them is seen alone: without SiLU the results are those of the same fp32 operations bit for
bit.  With it, u = 2^-24: the value is off by (|g| + 6) u of itself and the slope by (12 + 6 |g|) u, as for the small sizes; each product is a rounding more."""

import pytest

from operator_helpers import U, guarded, types
from paper_2001_00138_amd import binding as B
from test_gpu_fp8_products import KINDS, LARGE, whole
from test_gpu_rms import TINY

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def weights(torch, rows, k, squares, seed):
    """Whole numbers whose scales make sums of a few units"""
    codes, scales, values = whole(torch, rows, k, squares, seed)
    down = k.bit_length() // 2 + 6
    return codes, scales - down, values * 2.0 ** -down


def silu(z):
    return z / (1 + (-z).exp())


def near(got, want, off, kind):
    return bool(((got.double() - want).abs() <= off + U[kind] * (want.abs() + off) + TINY[kind]).all())


def random(torch, seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("rows,k,n", LARGE)
@pytest.mark.parametrize("squares", [False, True])
def test_linear(torch, rows, k, n, squares):
    (xc, xs, x), (wc, ws, w) = whole(torch, rows, k, False, 4), weights(torch, n, k, squares, 5)
    z, bias = (x @ w.t().contiguous()).float(), random(torch, 6, n)
    for kind in KINDS:
        t = types(torch)[kind]
        for act in ("none", "relu", "silu"):
            out, check = guarded(torch, (rows, n + 3), t)
            B.patdnn_fp8_linear(xc, xs, wc, ws, bias, out[:, :n], act=act)
            check()
            assert bool((out[:, n:] == 77).all())
            want = z + bias
            if act == "silu":
                assert near(out[:, :n], silu(want.double()), (want.double().abs() + 6) * u * silu(want.double()).abs(), kind)
            else:
                assert torch.equal(out[:, :n], (torch.relu(want) if act == "relu" else want).to(t))


@pytest.mark.parametrize("rows,k,n", LARGE)
@pytest.mark.parametrize("squares", [False, True])
def test_gated(torch, rows, k, n, squares):
    (xc, xs, x), (gc, gs, gate), (uc, us, up) = whole(torch, rows, k, False, 7), weights(torch, n, k, squares, 8), weights(torch, n, k, squares, 9)
    g, v = x @ gate.t().contiguous(), x @ up.t().contiguous()
    want = silu(g) * v
    off = (g.abs() + 8) * u * want.abs()
    for kind in KINDS:
        out, check = guarded(torch, (rows, n + 3), types(torch)[kind])
        B.patdnn_fp8_gated(xc, xs, gc, gs, uc, us, out[:, :n])
        check()
        assert bool((out[:, n:] == 77).all()) and near(out[:, :n], want, off, kind)
    codes, scales = B.patdnn_fp8_gated(xc, xs, gc, gs, uc, us, fp8=True)
    got = B.patdnn_fp8_dequantize(codes, scales, n).double()
    pieces = -(-n // 128)
    # half a code of the value, or of the smallest normal one of its block, whose largest takes 224 units and more
    top = torch.nn.functional.pad(want.abs() + off, (0, pieces * 128 - n)).view(rows, pieces, 128).amax(dim=2).repeat_interleave(128, dim=1)[:, :n]
    assert bool(((got - want).abs() <= off + torch.maximum(2.0 ** -4 * (want.abs() + off), 2.0 ** -10 * top / 223)).all())


@pytest.mark.parametrize("rows,k,n", LARGE)
@pytest.mark.parametrize("squares", [False, True])
def test_gated_backward(torch, rows, k, n, squares):
    (xc, xs, x), (gc, gs, gate), (uc, us, up) = whole(torch, rows, k, False, 10), weights(torch, n, k, squares, 11), weights(torch, n, k, squares, 12)
    g, v = x @ gate.t().contiguous(), x @ up.t().contiguous()
    s = 1 / (1 + (-g).exp())
    slope = s * (1 + g * (1 - s))
    for dkind in KINDS:
        on = torch.full((rows, n + 5), 9.0, dtype=types(torch)[dkind], device="cuda")
        on[:, :n] = random(torch, 13, rows, n).to(on.dtype)
        dh, d = on[:, :n], on[:, :n].double()
        dg, du = d * v * slope, d * g * s
        off = torch.cat(((d * v).abs() * (12 + 6 * g.abs()) * u + 2 * u * dg.abs(), (g.abs() + 7) * u * du.abs()), dim=1)
        for kind in KINDS:
            t = types(torch)[kind]
            for act in ("none", "silu"):
                out, check = guarded(torch, (rows, 2 * n + 3), t)
                B.patdnn_fp8_gated_backward(dh, xc, xs, gc, gs, uc, us, out[:, :2 * n], act=act)
                check()
                assert bool((out[:, 2 * n:] == 77).all())
                if act == "none":
                    assert torch.equal(out[:, :2 * n], torch.cat((dh.float() * v.float(), dh.float() * g.float()), dim=1).to(t))
                else:
                    assert near(out[:, :2 * n], torch.cat((dg, du), dim=1), off, kind)


# (nine to sixteen rows: below 1.25 * 2^30 products the kernel of few rows, tiles above)
@pytest.mark.parametrize("rows,k,n", [(9, 8200, 8190), (16, 8200, 8190), (12, 16200, 8190), (16, 16200, 8190), (9, 16200, 16400)])
def test_sixteen_rows_of_many_weights(torch, rows, k, n):
    test_linear(torch, rows, k, n, True)
