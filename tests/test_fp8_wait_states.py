"""The fp8 matrix instructions of kernel_fp8_tiles.hip stand in inline assembly, where the compiler does not see that a result needs time before it may be touched.  Here the built kernels'
own code is read: between such an instruction and anything but a matrix instruction that touches its sums lie 20 wait states, no other matrix instruction adds to the same sums within three of it, and
an operand that a vector instruction wrote is two states old.  Branches are followed."""

import os
import re
import subprocess

import pytest

from paper_2001_00138_amd import buildlib

LLVM = "/opt/rocm/llvm/bin"
OBJECT = os.path.join(buildlib.OBJ, "kernel_fp8_tiles.o")
SETTLED, APART, FRESH = 20, 3, 2


def _kernels(folder):
    """name -> [(address, mnemonic, operands, target of a branch)]"""
    run = lambda *a: subprocess.run([os.path.join(LLVM, a[0]), *a[1:]], check=True, capture_output=True, text=True, cwd=folder).stdout      # noqa: E731
    run("llvm-objcopy", "--dump-section", ".hip_fatbin=fat.bin", OBJECT, "copy.o")
    run("clang-offload-bundler", "-unbundle", "-type=o", "-targets=hipv4-amdgcn-amd-amdhsa--gfx950", "-input=fat.bin", "-output=device.o")
    kernels, code, start = {}, None, 0
    for line in run("llvm-objdump", "-d", "device.o").splitlines():
        head = re.match(r"^([0-9a-f]+) <(\w+)>:", line)
        if head:
            start, code = int(head[1], 16), kernels.setdefault(head[2], [])
            continue
        m = re.match(r"^\s+(\w+)(.*?)\s*// ([0-9A-F]+):", line)
        if m and code is not None:
            to = re.search(r"<\w+(?:\+0x([0-9a-f]+))?>", line) if m[1].startswith(("s_cbranch", "s_branch")) else None
            code.append((int(m[3], 16), m[1], m[2], start + int(to[1] or "0", 16) if to else None))
    return kernels


def _registers(text, kind):
    found = set()
    for one, low, high in re.findall(rf"\b{kind}(?:(\d+)|\[(\d+):(\d+)\])", text):
        found.update(range(int(low or one), int(high or one) + 1))
    return found


def _faults(code):
    """Walks the code in its order, and some way along each branch from where it is taken."""
    at = {c[0]: i for i, c in enumerate(code)}
    parsed = [(op, _registers(rest, "a"), [_registers(r, "v") for r in rest.split(",")], int(rest or 0, 0) if op == "s_nop" else 0) for _, op, rest, _ in code]
    bad, branches = [], []

    def walk(i, steps, now, products, sums, order, fresh):
        """sums, order: register -> when, and as which product, it was last added to; fresh: vector register -> when it was written."""
        whole = steps is None
        for _ in range(len(code) if whole else steps):
            if i >= len(code):
                break
            op, a, v, nop = parsed[i]
            if op.startswith("v_mfma_scale"):
                bad.extend((i, "again") for r in a if products - order.get(r, -99) <= APART)
                bad.extend((i, "operand") for part in v for r in part if now - fresh.get(r, -99) <= FRESH)
                products += 1
                for r in a:
                    sums[r], order[r] = now, products - 1
            else:
                bad.extend((i, "sums") for r in a if now - sums.get(r, -99) <= SETTLED)
                if op.startswith("v_") and v:
                    for r in v[0]:
                        fresh[r] = now
            now += 1 + nop
            to = code[i][3]
            if whole and to is not None:
                branches.append((at[to], now, products, dict(sums), dict(order), dict(fresh)))
            i += 1
            if op == "s_branch" and not whole:
                i = at[to]
            elif op in ("s_branch", "s_endpgm"):         # what follows is not reached from here
                if not whole:
                    break
                sums, order, fresh = {}, {}, {}
    walk(0, None, 0, 0, {}, {}, {})
    for to, *state in branches:
        walk(to, 60, *state)
    return bad


def test_the_reader_sees_what_it_looks_for():
    product = (0, "v_mfma_scale_f32_16x16x128_f8f6f4", " a[0:3], v[0:7], v[8:15], a[0:3], v16, v17 op_sel_hi:[0,0,0]", None)
    read, wait = (1, "v_accvgpr_read_b32", " v20, a3", None), lambda n: (2, "s_nop", f" {n}", None)
    end = (9, "s_endpgm", "", None)
    assert _faults([product, read, end]) and _faults([product, wait(15), wait(2), read, end]) and not _faults([product, wait(15), wait(3), read, end])
    assert _faults([product, product, end]) and not _faults([(3, "v_mov_b32", " v18, 0", None), product, end])
    assert _faults([(3, "v_mov_b32", " v16, 0", None), product, end]) and _faults([(3, "v_mov_b32", " v16, 0", None), wait(0), product, end])
    assert not _faults([(3, "v_mov_b32", " v16, 0", None), wait(1), product, end])
    # a branch back to a read of the sums
    assert _faults([(0, "v_accvgpr_read_b32", " v20, a3", None), wait(0), (4, "v_mfma_scale_f32_16x16x128_f8f6f4", product[2], None), (5, "s_cbranch_scc1", " 1", 0), end])


def test_wait_states(tmp_path):
    if not os.path.exists(OBJECT):
        pytest.skip("not built here")
    kernels = {k: v for k, v in _kernels(tmp_path).items() if any(op.startswith("v_mfma_scale") for _, op, _, _ in v)}
    assert len(kernels) >= 20
    for name, code in kernels.items():
        bad = _faults(code)
        assert not bad, (name, len(bad), [(why, *code[i][:3]) for i, why in bad[:5]])
