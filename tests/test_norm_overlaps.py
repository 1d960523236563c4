"""A group norm's small outputs may not share memory with its inputs, its workspace or one another: some workgroups still read what others write.
Refused before anything reaches a device."""

import ctypes

import pytest

from paper_2001_00138_amd import binding as B

L = B.lib
P = 1 << 20                        # stand for device addresses that no call gets as far as reading
DESC = dict(n=2, pixels=9, channels=8, groups=4, type=0, act=0, eps=1e-5, x_image=72, x_pixel=8, y_image=72, y_pixel=8, dy_image=72, dy_pixel=8)
X = 2 * 72 * 4                     # bytes of x


def _desc():
    return ctypes.byref(B.NormDesc(*(DESC[k] for k, _ in B.NormDesc._fields_)))


FORWARD = ["x", "gamma", "beta", "y", "mean", "rstd", "workspace"]
BACKWARD = ["dy", "x", "mean", "rstd", "gamma", "beta", "dx", "dgamma", "dbeta", "workspace"]


def _addresses(names):
    return {name: P + (i << 12) for i, name in enumerate(names)}


def _bytes(names, name):
    work = 4 * L().patdnn_group_norm_workspace_floats(_desc(), int(names is BACKWARD))
    return {"x": X, "y": X, "dy": X, "dx": X, "gamma": 32, "beta": 32, "dgamma": 32, "dbeta": 32, "mean": 32, "rstd": 32, "workspace": work}[name]


def _call(names, at):
    call = L().patdnn_group_norm if names is FORWARD else L().patdnn_group_norm_backward
    return call(_desc(), *(at[name] for name in names), 1 << 20, None)


@pytest.mark.parametrize("names,outputs", [(FORWARD, ["mean", "rstd"]), (BACKWARD, ["dgamma", "dbeta"])], ids=["forward", "backward"])
def test_small_outputs(names, outputs):
    for out in outputs:
        for other in names:
            if other == out:
                continue
            # the same, its last element, and one element into it
            for shift in (0, _bytes(names, other) - 4, 4 - _bytes(names, out)):
                at = _addresses(names)
                at[out] = at[other] + shift
                assert _call(names, at) == B.PATDNN_EINVAL, (out, other, shift)
                assert "overlap" in L().patdnn_last_error().decode(), (out, other, shift)


@pytest.mark.parametrize("names,inputs", [(FORWARD, ["gamma", "beta"]), (BACKWARD, ["mean", "rstd", "gamma", "beta"])], ids=["forward", "backward"])
def test_small_inputs(names, inputs):
    for name in inputs:
        for out in ("y", "workspace") if names is FORWARD else ("dx", "workspace"):
            at = _addresses(names)
            at[name] = at[out] + 4
            assert _call(names, at) == B.PATDNN_EINVAL, (name, out)
            assert "overlap" in L().patdnn_last_error().decode(), (name, out)
