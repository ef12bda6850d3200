"""The 8-bit GEMMs of 128 x 128 and 256 x 256 tiles issue their products as
instructions the compiler does not model, so it does not keep accesses of their
results clear of products still in the matrix pipe; the kernels' own order has
to.  The kernel for few rows uses the compiler's own products, and where a
branch lay between a product and the store of its result that compiler left too
few states.  Checked on the built library, over straight-line code and over
every branch."""

import os
import re
import subprocess

import pytest

import paper_2609_02846_amd as ue
from paper_2609_02846_amd import build as ue_build
from test_mfma_wait import LLVM, _code_objects

# States after which a VALU, LDS or memory instruction may touch the result of a
# product on 8-bit operands: of 8 passes (16 x 16 x 128) and 16 (32 x 32 x 64).
WAIT = {"gemm_fp8_kernel": 12, "gemm_fp8_wide_kernel": 20, "gemm_fp8_skinny_kernel": 12}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(ue.LIB_PATH):
        ue_build.build(verbose=False)
    tmp, found = tmp_path_factory.mktemp("isa"), {}
    for i, obj in enumerate(_code_objects(ue.LIB_PATH)):
        if not any(k.encode() in obj for k in WAIT):
            continue
        f = tmp / f"{i}.o"
        f.write_bytes(obj)
        name = None
        for line in subprocess.run([f"{LLVM}/llvm-objdump", "-d", str(f)], capture_output=True, text=True,
                                   check=True).stdout.splitlines():
            m = re.match(r"[0-9a-f]+ <(.+)>:$", line)
            if m:
                name = m.group(1) if any(k + "I" in m.group(1) for k in WAIT) else None
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


def _walk(code, order, wait, jump=None):
    """Instructions of ``order`` that touch a product's result too early."""
    pending, bad = [], []                        # (registers, states since)
    for i in order:
        text = code[i][1]
        mfma = text.startswith("v_mfma")
        regs = _registers(text)
        # a product may accumulate on another's result: the matrix pipe's own order
        if not mfma and any(regs & r for r, n in pending if n < wait):
            bad.append(text)
        pending = [(r, n + _states(text)) for r, n in pending if n < wait]
        if i != jump and text.startswith(("s_branch", "s_endpgm")):
            pending = []                         # what follows in memory does not follow in time
        if mfma:
            dest = re.match(r"\S+ ([va]\[\d+:\d+\])", text).group(1)
            pending.append((_registers(dest), 0))
    return bad


def test_products_land_before_they_are_read(kernels):
    # two formats, tilings and outputs; of the smaller tiles both scale kinds and heights
    assert sum("gemm_fp8_kernel" in n for n in kernels) == 32 and len(kernels) > 40
    for name, code in kernels.items():
        wait = next(w for k, w in WAIT.items() if k + "I" in name)
        at = {a: i for i, (a, _) in enumerate(code)}
        assert sum(t.startswith("v_mfma") for _, t in code) >= (1 if "skinny" in name else 32), name
        assert _walk(code, range(len(code)), wait) == [], name
        # every branch: the instructions before it, then those at its target
        for i, (a, text) in enumerate(code):
            m = re.match(r"s_c?branch\S* (\d+)", text)
            if m:
                offset = int(m.group(1))
                j = at[a + 4 + 4 * (offset - 0x10000 if offset >= 0x8000 else offset)]
                order = list(range(max(0, i - 60), i + 1)) + list(range(j, min(j + 60, len(code))))
                assert _walk(code, order, wait, i) == [], name
