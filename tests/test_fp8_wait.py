"""The 8-bit GEMM of 128 x 128 tiles issues its products as instructions the
compiler does not model, so it does not keep reads of their results clear of
products still in the matrix pipe; the kernel's own order has to.  Checked on
the built library, over straight-line code and over the loops' back edges."""

import os
import re
import subprocess

import pytest

import paper_2609_02846_amd as ue
from paper_2609_02846_amd import build as ue_build
from test_mfma_wait import LLVM, _code_objects

# v_mfma_f32_16x16x128_f8f6f4 on 8-bit operands takes 8 passes: a VALU, LDS or
# memory instruction may touch its result after this many others.
WAIT = 12


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(ue.LIB_PATH):
        ue_build.build(verbose=False)
    tmp, found = tmp_path_factory.mktemp("isa"), {}
    for i, obj in enumerate(_code_objects(ue.LIB_PATH)):
        if b"gemm_fp8_kernel" not in obj:
            continue
        f = tmp / f"{i}.o"
        f.write_bytes(obj)
        name = None
        for line in subprocess.run([f"{LLVM}/llvm-objdump", "-d", str(f)], capture_output=True, text=True,
                                   check=True).stdout.splitlines():
            m = re.match(r"[0-9a-f]+ <(.+)>:$", line)
            if m:
                name = m.group(1) if "gemm_fp8_kernel" in m.group(1) else None
                if name:
                    found[name] = []
            elif name and "//" in line:
                code, rest = line.split("//", 1)
                found[name].append((int(rest.split(":")[0], 16), code.strip()))
    return found


def _registers(text):
    """VGPRs and AGPRs an instruction names, as a set of (kind, number)."""
    out = set()
    for kind, one, lo, hi in re.findall(r"\b([va])(?:(\d+)\b|\[(\d+):(\d+)\])", text):
        out |= {(kind, n) for n in (range(int(lo), int(hi) + 1) if lo else [int(one)])}
    return out


def _states(text):
    m = re.match(r"s_nop (\d+)", text)
    return int(m.group(1)) + 1 if m else 1


def _walk(code, order):
    """Instructions of ``order`` that touch a product's result too early."""
    pending, bad = [], []                        # (registers, states since)
    for i in order:
        text = code[i][1]
        mfma = text.startswith("v_mfma")
        regs = _registers(text)
        # a product may accumulate on another's result: the matrix pipe's own order
        if not mfma and any(regs & r for r, n in pending if n < WAIT):
            bad.append(text)
        pending = [(r, n + _states(text)) for r, n in pending if n < WAIT]
        if mfma:
            dest = re.match(r"\S+ ([va]\[\d+:\d+\])", text).group(1)
            pending.append((_registers(dest), 0))
    return bad


def test_products_land_before_they_are_read(kernels):
    assert len(kernels) == 16                    # two formats, scale kinds, tilings and outputs
    for name, code in kernels.items():
        at = {a: i for i, (a, _) in enumerate(code)}
        assert sum(t.startswith("v_mfma") for _, t in code) >= 32, name
        assert not any("scratch_" in t for _, t in code), name
        assert _walk(code, range(len(code))) == [], name
        # every backward branch: the loop's last instructions, then its first
        for i, (a, text) in enumerate(code):
            m = re.match(r"s_c?branch\S* (\d+)", text)
            if m and int(m.group(1)) >= 0x8000:
                target = a + 4 + 4 * (int(m.group(1)) - 0x10000)
                j = at[target]
                assert _walk(code, list(range(max(0, i - 60), i + 1)) + list(range(j, min(j + 60, len(code))))) == [], name
