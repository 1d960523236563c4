"""Group norm at sizes where pixels and channels are dealt out to lanes in uncommon ways, against the oracle in 64 bits.  Tolerances as in test_gpu_norm.py."""

import pytest

import test_gpu_norm as norm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


# many images and chunks, groups that are no whole runs of 16 bytes: runs of a lane hold channels of two groups
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(64, 49, 640, 32), (64, 49, 320, 32), (36, 110, 896, 32), (80, 49, 384, 32), (70, 154, 384, 32), (64, 110, 896, 32)])
def test_runs_across_groups(torch, shape, kind):
    norm._both(torch, shape, kind, ["none", "relu", "silu"][(shape[0] + shape[1] + shape[2]) % 3])


# one pixel more than whole rows of lanes, and its neighbours
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(64, 127, 256, 32), (64, 128, 256, 32), (64, 129, 256, 32), (64, 257, 256, 32), (128, 641, 128, 16)])
def test_pixels_beside_whole_rows_of_lanes(torch, shape, kind):
    norm._both(torch, shape, kind, ["none", "relu", "silu"][(shape[0] + shape[1] + shape[2]) % 3])
