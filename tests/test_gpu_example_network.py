"""The example network: each step against the oracle on the tensors that the step before it left, so that a code which rounds the other way in one
step does not hide what the next one does."""

import numpy as np
import pytest

from operator_helpers import U, doubles
from oracle import operators as oo
from paper_2001_00138_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 5])
def test_every_step(n):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2001_00138_amd.examples import pruned_network as pn
    net = pn.Network(side=14, seed=3)
    x = torch.randn(n, pn.WIDTHS[0], 14, 14, device="cuda")
    steps = []
    logits = net(x, steps)
    assert logits.shape == (n, pn.CLASSES)
    at = 0

    def layer(rows, w, scales, bias, act):
        cols = rows.shape[1]
        q = B.patdnn_mxfp4_quantize(rows)
        values = oo.mxfp4_values(*(t.cpu().numpy() for t in q), cols)
        y, size = oo.linear(values, oo.mxfp4_values(w.cpu().numpy(), scales.cpu().numpy(), cols), doubles(bias), act)
        return y, 1.1 * (cols + 2) * U["f32"] * size
    for block, (_, gamma, beta, (w, scales, bias)) in enumerate(net.blocks):
        names = [s[0] for s in steps[at:at + 7]]
        assert names == ["conv", "last", "norm", "mean", "rstd", "pointwise", "first"]
        conv, last, norm, mean, rstd, pointwise, first = (s[1] for s in steps[at:at + 7])
        at += 7
        assert torch.equal(last, conv.permute(0, 2, 3, 1).half())
        y, m, r = oo.group_norm(doubles(last), pn.GROUPS, doubles(gamma), doubles(beta), 1e-5, "silu")
        assert (np.abs(doubles(norm) - y) <= 1e-5 * np.abs(y).max() + U["f16"] * np.abs(y) * 1.01 + 2.0 ** -24).all()
        assert np.abs(doubles(mean) - m).max() <= 1e-5 and (np.abs(doubles(rstd) - r) <= 1e-5 * r).all()
        dy = torch.randn_like(norm)
        dx, dgamma, dbeta = net.normalisation_gradients(block, last, mean, rstd, dy)
        wx, wg, wb = oo.group_norm_backward(doubles(dy), doubles(last), doubles(mean), doubles(rstd), pn.GROUPS, doubles(gamma), doubles(beta), "silu")
        assert (np.abs(doubles(dx) - wx) <= 1e-5 * np.abs(wx).max() + U["f16"] * np.abs(wx) * 1.01 + 2.0 ** -24).all()
        assert np.abs(doubles(dgamma) - wg).max() <= 1e-5 * np.abs(wg).max() and np.abs(doubles(dbeta) - wb).max() <= 1e-5 * np.abs(wb).max()
        y, allowed = layer(norm.view(-1, norm.shape[-1]), w, scales, bias, "relu")
        got = doubles(pointwise).reshape(y.shape)
        assert (np.abs(got - y) <= allowed + U["f16"] * np.abs(y) * 1.01 + 2.0 ** -24).all()
        assert torch.equal(first, pointwise.permute(0, 3, 1, 2).float())
    pool = steps[at][1]
    y, allowed = layer(pool.view(n, -1), *net.classifier, "none")
    assert (np.abs(doubles(logits) - y) <= allowed).all()
    net.close()
