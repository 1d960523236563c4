"""A workspace that the binding of the operators allocates is held until the call that uses it has returned: the library is replaced by
one that looks whether its workspace is still owned.  (Freed earlier, another thread on the stream may be given the memory before the kernels are launched.)"""

import weakref

import numpy as np
import pytest
import torch

from paper_2001_00138_amd import binding as B


class OnDevice(torch.Tensor):
    """A host tensor that says that it is a device tensor."""
    is_cuda = property(lambda self: True)


def _device(t):
    return t.as_subclass(OnDevice)


class Library:
    """Sizes as the caller of the fixture wants them; calls that note whether the allocation that holds their workspace is alive."""

    def __init__(self, size, made):
        self.size, self.made, self.alive = size, made, []

    def _look(self, workspace, needs):
        whole = [array for array in (ref() for ref in self.made)
                 if array is not None and array.ctypes.data <= workspace and workspace + needs <= array.ctypes.data + array.nbytes]
        self.alive.append(len(whole) == 1)
        return B.PATDNN_OK

    def patdnn_group_norm_workspace_floats(self, desc, backward):
        return self.size

    def patdnn_mxfp4_linear_workspace_bytes(self, desc):
        return self.size

    def patdnn_group_norm(self, *args):
        return self._look(args[7], 4 * self.size)

    def patdnn_group_norm_backward(self, *args):
        return self._look(args[10], 4 * self.size)

    def patdnn_mxfp4_linear(self, *args):
        return self._look(args[7], self.size)


@pytest.fixture(params=[100, 1 << 16, (1 << 16) + 1, 1 << 20])
def library(request, monkeypatch):
    made = []

    def new(shape, dtype, like, stream):
        array = np.empty(int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size(), np.uint8)
        made.append(weakref.ref(array))
        return _device(torch.from_numpy(array).view(dtype).view(shape))
    fake = Library(request.param, made)
    monkeypatch.setattr(B, "lib", lambda: fake)
    monkeypatch.setattr(B, "_new", new)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: None)
    return fake


def test_the_fixture_sees_a_workspace_that_is_gone(library):
    t = B._new((library.size,), torch.float32, None, None)
    at = t.data_ptr()
    assert library._look(at, 4 * library.size) == B.PATDNN_OK and library.alive == [True]
    del t
    library._look(at, 4 * library.size)
    assert library.alive == [True, False]


def test_group_norm(library):
    x = _device(torch.zeros(2, 3, 3, 8))
    given = lambda: _device(torch.zeros(2, 4))                 # noqa: E731
    for more in ({}, {"mean": given()}, {"rstd": given()}, {"mean": given(), "rstd": given()}, {"out": _device(torch.zeros(2, 3, 3, 8))}):
        B.patdnn_group_norm(x, 4, **more)
        assert library.alive.pop(), more


def test_group_norm_backward(library):
    x, mean = _device(torch.zeros(2, 3, 3, 8)), _device(torch.zeros(2, 4))
    given = lambda: _device(torch.zeros(8))                    # noqa: E731
    for more in ({}, {"dgamma": given()}, {"dbeta": given()}, {"dgamma": given(), "dbeta": given()}):
        B.patdnn_group_norm_backward(x, x, mean, mean, 4, **more)
        assert library.alive.pop(), more


def test_a_workspace_of_the_callers(library):
    work = B._new((library.size,), torch.float32, None, None)
    x, mean = _device(torch.zeros(2, 3, 3, 8)), _device(torch.zeros(2, 4))
    B.patdnn_group_norm(x, 4, workspace=work)
    B.patdnn_group_norm_backward(x, x, mean, mean, 4, workspace=work)
    assert library.alive == [True, True]


def test_linear(library):
    x, w = _device(torch.zeros(20, 40)), _device(torch.zeros(8, 64, dtype=torch.uint8))
    B.patdnn_mxfp4_linear(x, w, _device(torch.zeros(8, 4, dtype=torch.uint8)))
    assert library.alive == [True]
