"""The compiler reserves m0 and cannot be told that inline assembly changes it, so assembly that does leaves m0 as it found it."""

import glob
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2001_00138_amd", "csrc")
FILES = sorted(os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.hpp")))


def _assembly(text):
    """The instructions of each asm statement, in order."""
    text = re.sub(r"//.*", "", text)
    for m in re.finditer(r'\basm\s*(?:volatile)?\s*\(\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', text):
        whole = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', m.group(1)))
        yield [i.strip() for i in re.split(r"\\n|\\t|;", whole) if i.strip()]


@pytest.mark.parametrize("name", FILES)
def test_m0_is_left_as_it_was(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    for lines in _assembly(text):
        writes = [i for i in lines if re.match(r"s_\w+ m0\b", i)]
        if not writes:
            continue
        saved = re.match(r"s_mov_b32 (\S+), m0$", lines[0])
        assert saved and lines[-1] == f"s_mov_b32 m0, {saved.group(1)}" and lines.count(lines[0]) == 1, lines


def test_the_statements_are_found():
    with open(os.path.join(CSRC, "kernel_linear_tiles.hip")) as f:
        found = [lines for lines in _assembly(f.read()) if any("lds" in i and i.startswith("buffer_load") for i in lines)]
    assert len(found) == 2
