"""A scalar register that a vector instruction wrote (a lane read out, a
comparison) may be taken by a memory instruction five states later at the
earliest.  The compiler keeps to that for the instructions that it models, not
for loads written as inline assembly, whose buffer descriptor it may have just
brought back from a spilled lane.  Checked on the built library, in straight
lines and over every branch."""

import os
import re
import subprocess

import paper_2609_02846_amd as ue
from paper_2609_02846_amd import build as ue_build
from test_mfma_wait import LLVM, _code_objects

WAIT = 5
MEMORY = ("buffer_", "global_", "scratch_", "flat_")


def _scalars(text):
    """Scalar registers an instruction's operands name."""
    out = set()
    for one, lo, hi in re.findall(r"\bs(?:(\d+)\b|\[(\d+):(\d+)\])", text):
        out |= set(range(int(lo), int(hi) + 1) if lo else [int(one)])
    return out


def _written(text):
    """Scalar registers that a vector instruction writes."""
    op, _, rest = text.partition(" ")
    args = rest.split(",")
    if op.startswith(("v_readfirstlane", "v_readlane")) or op.startswith("v_cmp"):
        return _scalars(args[0])
    return _scalars(args[1]) if "_co_" in op and len(args) > 1 else set()


def _states(text):
    m = re.match(r"s_nop (\d+)", text)
    return int(m.group(1)) + 1 if m else 1


def _walk(code, order):
    """Memory instructions of ``order`` that take a register too early."""
    age, bad = {}, []
    for i in order:
        text = code[i][1]
        if text.startswith(MEMORY) and _scalars(text) & set(age):
            bad.append(text)
        n = _states(text)
        age = {r: a + n for r, a in age.items() if a + n < WAIT}
        if text.startswith("s_") and " " in text and not text.startswith(("s_nop", "s_cmp", "s_bitcmp")):
            for r in _scalars(text.split(" ", 1)[1].split(",")[0]):
                age.pop(r, None)                     # a scalar instruction's result instead
        age.update({r: 0 for r in _written(text)})
    return bad


def _functions(path, tmp):
    for i, obj in enumerate(_code_objects(path)):
        f = tmp / f"{i}.o"
        f.write_bytes(obj)
        name, code = None, []
        for line in subprocess.run([f"{LLVM}/llvm-objdump", "-d", str(f)], capture_output=True, text=True,
                                   check=True).stdout.splitlines():
            m = re.match(r"[0-9a-f]+ <(.+)>:$", line)
            if m:
                if code:
                    yield name, code
                name, code = m.group(1), []
            elif name and "//" in line:
                text, rest = line.split("//", 1)
                code.append((int(rest.split(":")[0], 16), text.strip()))
        if code:
            yield name, code


def test_the_rule_sees_a_load_that_comes_too_early():
    line = lambda *text: list(enumerate(text))  # noqa: E731
    early = line("v_readlane_b32 s8, v1, 3", "s_add_u32 m0, s5, 0", "s_nop 0", "buffer_load_dwordx4 v7, s[8:11], s6 offen lds")
    assert _walk(early, range(4)) and not _walk(early[:2] + line("s_nop 3")[:1] + early[3:], range(4))
    assert not _walk(early[:1] + line("s_mov_b32 s8, 0") + early[3:], range(3))
    assert _walk(line("v_cmp_lt_i32_e64 s[6:7], 0, v1", "global_load_dword v1, v2, s[6:7]"), range(2))


def test_memory_instructions_come_after_their_scalars(tmp_path):
    if not os.path.exists(ue.LIB_PATH):
        ue_build.build(verbose=False)
    seen, bad = 0, {}
    for name, code in _functions(ue.LIB_PATH, tmp_path):
        at = {a: i for i, (a, _) in enumerate(code)}
        orders = [range(len(code))]
        for i, (a, text) in enumerate(code):
            m = re.match(r"s_c?branch\S* (\d+)", text)
            if m:
                offset = int(m.group(1))
                j = at[a + 4 + 4 * (offset - 0x10000 if offset >= 0x8000 else offset)]
                orders.append([*range(max(0, i - WAIT), i + 1), *range(j, min(j + WAIT, len(code)))])
        for order in orders:
            found = _walk(code, order)
            if found:
                bad.setdefault(name, []).extend(found)
        seen += 1
    assert seen > 200 and not bad, bad
