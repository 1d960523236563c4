"""The binding of the feed-forward block's operators: workspaces that it allocates are owned until the call has returned, calls are made with the tensors' device
current, and tensors of two devices, of other types or shapes are refused."""

import numpy as np
import pytest
import torch

from paper_2001_00138_amd import binding as B


class OnDevice(torch.Tensor):
    """A host tensor that says that it is one of device number `INDEX`."""
    INDEX = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return type(self).INDEX


class OnAnother(OnDevice):
    INDEX = 1


def _device(t, cls=OnDevice):
    return t.as_subclass(cls)


class Library:
    """Workspaces of `size`; calls that note whether what they get is owned by one of `made`, and which device is current."""

    def __init__(self, size, made, current):
        self.size, self.made, self.current, self.calls = size, made, current, []

    def __getattr__(self, name):
        if name.endswith(("_bytes", "_floats")):
            return lambda *args: self.size

        def call(*args):
            self.calls.append((name, self.current[-1]))
            if name in ("patdnn_fp8_linear", "patdnn_fp8_gated", "patdnn_fp8_gated_backward", "patdnn_rms_norm_backward") and self.size:
                at, size = args[-3], args[-2]
                assert size >= self.size and any(a() is not None and a().data_ptr() <= at < a().data_ptr() + a().numel() * a().element_size() for a in self.made)
            return B.PATDNN_OK
        return call


@pytest.fixture(params=[0, 4096])
def library(request, monkeypatch):
    import weakref
    made, current = [], [0]

    def new(shape, dtype, like, stream):
        t = torch.zeros(shape, dtype=dtype).as_subclass(type(like))
        made.append(weakref.ref(t))
        return t

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            current.append(self.index)

        def __exit__(self, *_):
            current.pop()
    lib = Library(request.param, made, current)
    monkeypatch.setattr(B, "lib", lambda: lib)
    monkeypatch.setattr(B, "_new", new)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[-1], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "device", Device)
    return lib


def _calls(cls):
    x = _device(torch.zeros(3, 256), cls)
    c, s = _device(torch.zeros(3, 256, dtype=torch.uint8), cls), _device(torch.zeros(3, 2, dtype=torch.uint8), cls)
    r = _device(torch.zeros(3), cls)
    B.patdnn_fp8_quantize(x)
    B.patdnn_fp8_quantize(x, blocks="squares", transposed=True)
    B.patdnn_fp8_dequantize(c, s, 256)
    B.patdnn_rms_norm(x, residual=x, fp8=True)
    B.patdnn_rms_norm_backward(x, x, r)
    B.patdnn_fp8_linear(c, s, c, s)
    B.patdnn_fp8_gated(c, s, c, s, c, s, fp8=True)
    B.patdnn_fp8_gated_backward(_device(torch.zeros(3, 3), cls), c, s, c, s, c, s)


@pytest.mark.parametrize("cls", [OnDevice, OnAnother])
def test_device_and_workspace(library, cls):
    _calls(cls)
    assert len(library.calls) == 8 and all(device == cls.INDEX for _, device in library.calls) and library.current == [0]


def test_refusals(library):
    x = _device(torch.zeros(3, 256))
    c, s = _device(torch.zeros(3, 256, dtype=torch.uint8)), _device(torch.zeros(3, 2, dtype=torch.uint8))
    other = _device(torch.zeros(3, 2, dtype=torch.uint8), OnAnother)
    cases = [("one device", lambda: B.patdnn_fp8_linear(c, other, c, s)), ("one device", lambda: B.patdnn_rms_norm(x, residual=_device(torch.zeros(3, 256), OnAnother))),
             ("uint8 or float8", lambda: B.patdnn_fp8_linear(x, s, c, s)), ("whole pieces", lambda: B.patdnn_fp8_linear(c[:, :200], s, c, s)),
             ("x_scales must be", lambda: B.patdnn_fp8_linear(c, s[:, :1], c, s)), ("scales of the weights must be", lambda: B.patdnn_fp8_linear(c, s, c, s[:2])),
             ("one length", lambda: B.patdnn_fp8_linear(c, s, _device(torch.zeros(3, 128, dtype=torch.uint8)), s)),
             ("same number", lambda: B.patdnn_fp8_gated(c, s, c, s, c[:2], s[:2])), ("output must be", lambda: B.patdnn_fp8_linear(c, s, c, s, None, x)),
             ("dtype is for", lambda: B.patdnn_fp8_gated(c, s, c, s, c, s, fp8=True, dtype=torch.float32)), ("scales are for", lambda: B.patdnn_fp8_gated(c, s, c, s, c, s, scales=s)),
             ("scales are for", lambda: B.patdnn_rms_norm(x, scales=s)), ("residual must be", lambda: B.patdnn_rms_norm(x, residual=x.double())),
             ("dy must have", lambda: B.patdnn_rms_norm_backward(x[:2], x, _device(torch.zeros(3)))), ("columns are not", lambda: B.patdnn_fp8_dequantize(c, s, 128)),
             ("act must be", lambda: B.patdnn_fp8_linear(c, s, c, s, act="gelu")), ("dh must be", lambda: B.patdnn_fp8_gated_backward(x, c, s, c, s, c, s)),
             ("adjacent", lambda: B.patdnn_rms_norm(x.t())), ("2-d", lambda: B.patdnn_fp8_quantize(x.view(3, 2, 128)))]
    for word, call in cases:
        with pytest.raises(ValueError, match=word):
            call()
    assert not library.calls
    assert np.prod(B.patdnn_fp8_linear(c, s, c, s).shape) == 9
