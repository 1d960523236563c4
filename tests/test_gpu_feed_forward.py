"""The operators of a feed-forward block together, as the example calls them: every step against the oracle on what the step before gave, forward and backward;
captured into a graph, on another stream, from two streams at once.

Tolerances as in the tests of the single operators; codes of a step are half a code away at most, and the next step takes them as they are."""

import numpy as np
import pytest

from oracle import feed_forward as ff
from oracle.operators import activation, activation_slope
from operator_helpers import U, doubles
from paper_2001_00138_amd import binding as B
from paper_2001_00138_amd.examples.feed_forward import Block
from test_gpu_fp8_products import near, sums_of
from test_gpu_rms import TINY, chain, check_codes

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _values(codes, scales, cols):
    return ff.fp8_values(codes.cpu().numpy(), scales.cpu().numpy(), cols)


@pytest.mark.parametrize("rows,width,hidden", [(1, 256, 384), (37, 200, 300), (150, 384, 136)])
def test_forward_and_backward_step_by_step(torch, rows, width, hidden):
    block = Block(width, hidden, seed=rows)
    torch.manual_seed(rows)
    x, residual, dout, dstream = (torch.randn(rows, width, device="cuda").bfloat16() for _ in range(4))
    kept = {}
    out, stream = block(x, residual, kept)
    gamma = doubles(block.gamma)
    y, s, rstd = ff.rms_norm(doubles(x), doubles(residual), gamma, block.eps)
    rel = (chain(width) / 2 + 8) * u
    assert (np.abs(doubles(stream) - s) <= (U["bf16"] + 2 * u) * np.abs(s) + TINY["bf16"]).all()
    check_codes(kept["codes"].cpu().numpy(), kept["scales"].cpu().numpy(), y, rel * np.abs(y))
    normed = _values(kept["codes"], kept["scales"], width)
    gate, up = _values(block.gate, block.gate_scales, width), _values(block.up, block.up_scales, width)
    (g, eg), (v, ev) = sums_of(normed, gate, "fp8"), sums_of(normed, up, "fp8")
    value = activation(g, "silu")
    evalue = 1.1 * eg + (np.abs(g) + 6) * u * np.abs(value)
    check_codes(kept["h"].cpu().numpy(), kept["h_scales"].cpu().numpy(), value * v, evalue * (np.abs(v) + ev) + np.abs(value) * ev + 2 * u * np.abs(value * v))
    h = _values(kept["h"], kept["h_scales"], hidden)
    z, off = sums_of(h, _values(*block.down8, hidden), "bf16")
    assert near(doubles(out), z, off, "bf16")

    got = block.gradients(kept, dout, dstream)
    dout8 = B.patdnn_fp8_quantize(dout)
    dh, edh = sums_of(_values(*dout8, width), _values(*block.down_t, width), "bf16")
    on_gpu = B.patdnn_fp8_linear(*dout8, *block.down_t, dtype=torch.bfloat16)
    assert near(doubles(on_gpu), dh, edh, "bf16")
    # the weights' codes turned are the codes of the weights turned
    assert torch.equal(block.down_t[0][:, :width], block.down8[0][:, :hidden].t())
    d_both = B.patdnn_fp8_gated_backward(on_gpu, kept["codes"], kept["scales"], block.gate, block.gate_scales, block.up, block.up_scales)
    (g, eg), (v, ev) = sums_of(normed, gate, "bf16"), sums_of(normed, up, "bf16")
    slope, d = activation_slope(g, "silu"), np.abs(doubles(on_gpu))
    dg, du = ff.gated_backward(doubles(on_gpu), g, v, "silu")
    eslope = 0.5 * eg + (12 + 6 * np.abs(g)) * u
    off = np.hstack((d * (ev * (np.abs(slope) + eslope) + np.abs(v) * eslope) + 2 * u * np.abs(dg), d * evalue + u * np.abs(du)))
    assert near(doubles(d_both), np.hstack((dg, du)), off, "bf16")
    both8 = B.patdnn_fp8_quantize(d_both)
    dn, edn = sums_of(_values(*both8, 2 * hidden), _values(*block.both_t, 2 * hidden), "bf16")
    d_normed = B.patdnn_fp8_linear(*both8, *block.both_t, dtype=torch.bfloat16)
    assert near(doubles(d_normed), dn, edn, "bf16")
    dx, dgamma = ff.rms_norm_backward(doubles(d_normed), doubles(stream), doubles(kept["rstd"]), gamma, doubles(dstream))
    rr, xh = doubles(kept["rstd"])[:, None], np.abs(doubles(stream) * doubles(kept["rstd"])[:, None])
    dd = np.abs(doubles(d_normed) * gamma)
    off = u * (4 * rr * dd + rr * xh * (dd * xh).mean(axis=1, keepdims=True) * (2 * chain(width) + 12) + 2 * np.abs(doubles(dstream)))
    assert near(doubles(got["x"]), dx, off, "bf16")
    assert (np.abs(doubles(got["gamma"]) - dgamma) <= 70 * u * (np.abs(doubles(d_normed)) * xh).sum(axis=0)).all()
    turned = lambda t: _values(*B.patdnn_fp8_quantize(t, transposed=True), rows)      # noqa: E731
    for name, a, b in (("both", turned(d_both), turned(torch.from_numpy(normed).cuda().bfloat16())), ("down", turned(dout), turned(torch.from_numpy(h).cuda().bfloat16()))):
        z, off = sums_of(a, b, "f32")
        assert near(doubles(got[name]), z, off, "f32")


def test_no_rows(torch):
    block = Block(200, 300)
    x = torch.empty(0, 200, device="cuda", dtype=torch.bfloat16)
    kept = {}
    out, stream = block(x, x, kept)
    got = block.gradients(kept, out, stream)
    assert out.shape == (0, 200) and got["x"].shape == (0, 200) and all(bool((got[k] == 0).all()) for k in ("gamma", "both", "down"))


@pytest.mark.parametrize("rows", [1, 100])
def test_graph_and_streams(torch, rows):
    """A pass and its gradients in a graph, replayed while the program goes on eagerly; then from two streams at once, each with its own tensors."""
    block = Block(512, 640)
    x, residual, dout = (torch.randn(rows, 512, device="cuda").bfloat16() for _ in range(3))
    held = {}

    def call():
        kept = {}
        out, stream = block(x, residual, kept)
        held["out"] = [out, stream, *block.gradients(kept, dout, stream).values()]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    captured = held["out"]
    for i in range(3):
        x.normal_(0, 1 + i)
        for t in captured:
            t.fill_(99)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, held["out"]))
    inputs = [torch.randn(rows, 512, device="cuda").bfloat16() for _ in range(2)]
    want = [block(t, residual)[0].clone() for t in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = [[], []]
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                results[k].append(block(inputs[k], residual)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(r, want[k]) for k in range(2) for r in results[k])


def test_main_runs(torch, capsys):
    from paper_2001_00138_amd.examples import feed_forward
    feed_forward.main()
    assert "us a pass" in capsys.readouterr().out
