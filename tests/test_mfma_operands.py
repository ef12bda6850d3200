"""A product may read a register two states after a vector instruction wrote
it.  The compiler keeps to that for its own products, and for those written as
inline assembly the kernels' order has to.  Checked on the built library, in
straight lines and over every branch."""

import os
import re

import paper_2609_02846_amd as ue
from paper_2609_02846_amd import build as ue_build
from test_fp8_wait import _registers, _states
from test_sgpr_wait import _functions

WAIT = 2


def _walk(code, order):
    """Products of ``order`` that read a register too early."""
    age, bad = {}, []
    for i in order:
        text = code[i][1]
        op, _, args = text.partition(" ")
        if op.startswith("v_mfma") and _registers(args.split("],", 1)[1]) & set(age):
            bad.append(text)
        n = _states(text)
        age = {r: a + n for r, a in age.items() if a + n < WAIT}
        if op.startswith("v_") and not op.startswith(("v_mfma", "v_cmp", "v_readfirstlane", "v_readlane")):
            age.update({r: 0 for r in _registers(args.split(",")[0])})
    return bad


def test_the_rule_sees_a_product_that_comes_too_early():
    product = "v_mfma_f32_16x16x128_f8f6f4 v[0:3], v[8:15], v[16:23], 0"
    line = lambda *text: list(enumerate(text))  # noqa: E731
    assert _walk(line("v_mov_b32_e32 v9, v1", product), range(2))
    assert _walk(line("v_mov_b64_e32 v[22:23], v[4:5]", "s_nop 0", product), range(3))
    assert not _walk(line("v_mov_b32_e32 v9, v1", "s_nop 1", product), range(3))
    assert not _walk(line("v_mov_b32_e32 v1, v9", product), range(2))


def test_products_come_after_their_operands(tmp_path):
    if not os.path.exists(ue.LIB_PATH):
        ue_build.build(verbose=False)
    products, bad = 0, {}
    for name, code in _functions(ue.LIB_PATH, tmp_path):
        n = sum(t.startswith("v_mfma") for _, t in code)
        if n == 0:
            continue
        products += n
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
    assert products > 10000 and not bad, bad
