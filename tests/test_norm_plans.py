"""What the library would launch for a group norm, over many sizes: a lane holds all of its pixels' runs, and lanes that keep one statistic
for their channels have channels of one group only.  Reads the plan; nothing is launched."""

import ctypes
import random

import pytest

from paper_2001_00138_amd import binding as B

BYTES = {0: 4, 1: 2, 2: 2}


def _plan(n, pixels, c, groups, kind, backward):
    image = pixels * c
    d = B.NormDesc(n, pixels, c, groups, kind, 0, 1e-5, image, c, image, c, image, c)
    out = (ctypes.c_int32 * 8)()
    assert B.lib().patdnn_internal_norm_plan(ctypes.byref(d), int(backward), out) == B.PATDNN_OK
    return dict(zip(("v", "runs", "room", "one", "threads", "rows", "chunk", "lds"), out))


def _shapes():
    """The sizes at which lanes and pixels are dealt out differently, then sizes all over the range."""
    for c, groups in [(640, 32), (320, 32), (896, 32), (384, 32), (960, 32), (96, 32), (480, 24), (256, 32), (512, 16), (64, 8), (32, 4), (1024, 32), (60, 4), (36, 4)]:
        for n in (1, 6, 36, 64, 300):
            for pixels in [*range(1, 40), 49, 63, 64, 65, 110, 127, 128, 129, 154, 196, 255, 256, 257, 784, 1023, 1024, 1025, 1663, 1664, 1665, 3136, 4096, 4097]:
                yield n, pixels, c, groups
    rng = random.Random(20)
    for _ in range(20000):
        groups = rng.choice([1, 2, 3, 4, 8, 16, 24, 32, 48])
        per = int(2 ** rng.uniform(0, 10))
        yield int(2 ** rng.uniform(0, 9)), int(2 ** rng.uniform(0, 14)), groups * per, groups


@pytest.fixture(scope="module")
def shapes():
    return list(_shapes())


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_one_statistic_for_channels_of_one_group(shapes, kind, backward):
    held = 0
    for n, pixels, c, groups in shapes:
        p = _plan(n, pixels, c, groups, kind, backward)
        if not p["v"]:
            continue
        held += 1
        # what the launch takes: where channels of a run are of several groups, the backward kernel exists for so many runs only
        several = not p["one"] and (not backward or p["room"] <= 4 * (BYTES[kind] // 2))
        assert several or (c // groups) % p["v"] == 0, (n, pixels, c, groups, p)
    assert held > 1000


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_a_lane_has_room_for_its_runs(shapes, kind, backward):
    held = 0
    for n, pixels, c, groups in shapes:
        p = _plan(n, pixels, c, groups, kind, backward)
        if not p["v"]:
            continue
        held += 1
        case = (n, pixels, c, groups, p)
        assert p["rows"] * p["runs"] >= pixels > p["rows"] * (p["runs"] - 1) and p["runs"] <= p["room"], case
        assert p["chunk"] % p["v"] == 0 and p["chunk"] % (c // groups) == 0 and p["rows"] * (p["chunk"] // p["v"]) <= p["threads"], case
        assert p["threads"] % 64 == 0 and p["threads"] <= 1024 and p["lds"] <= 160 * 1024, case
    assert held > 1000
