"""The 8-bit GEMM of 256 x 256 tiles waits for a stage by the number of loads
that may still be out: one, as the last load of each turn (a line for the L2) is
no part of a stage.  The first turn's wait needs as many loads before it as any
other's, or a stage's last scale codes may be read before they are there.
Checked on the built library."""

import pytest

from test_fp8_wait import kernels  # noqa: F401

STAGE = 18                                       # loads: 16 of rows, 2 of scale codes


def test_each_wait_leaves_out_only_the_line_ahead(kernels):  # noqa: F811
    wide = {n: [t for _, t in code] for n, code in kernels.items() if "gemm_fp8_wide_kernelI" in n}
    assert len(wide) == 8
    for name, code in wide.items():
        waits = [i for i, t in enumerate(code) if t.startswith("s_waitcnt") and "vmcnt(1)" in t]
        assert len(waits) == 1, name
        # from the wait for all of stage 0 on: stage 1 and the line ahead of it
        first = code.index("s_barrier")
        before = [t for t in code[first:waits[0]] if t.startswith("buffer_load")]
        assert len(before) == STAGE + 1, name
        assert [t.split()[0] for t in before[-3:]] == ["buffer_load_ubyte"] * 2 + ["buffer_load_dword"], name
        # and within a turn, in the same order
        turn = [t for t in code[waits[0]:] if t.startswith("buffer_load")]
        assert len(turn) == STAGE + 1, name
        assert [t.split()[0] for t in turn[-3:]] == ["buffer_load_ubyte"] * 2 + ["buffer_load_dword"], name
