"""Direct loads to LDS take their address from m0, which the compiler reserves
but does not track: between the statement that writes it and one that takes it
anything could change it.  The 8-bit products' kernels write and take it in one
statement.  Checked on the built library: right before each such load, with the
one state between that the write needs, stands a write of m0."""

import re

from test_fp8_wait import kernels  # noqa: F401


def test_each_direct_load_follows_its_own_write_of_m0(kernels):  # noqa: F811
    total = 0
    for name, code in kernels.items():
        text = [t for _, t in code]
        loads = [i for i, t in enumerate(text) if t.startswith("buffer_load") and t.endswith(" lds")]
        assert len(loads) >= 6, name
        for i in loads:
            assert re.match(r"s_(mov_b32|add_u32|add_i32) m0,", text[i - 2]), (name, text[i - 2:i + 1])
            assert not re.search(r"\bm0\b", text[i - 1]), (name, text[i - 2:i + 1])
        # and nothing else has a use for it
        others = [t for i, t in enumerate(text) if re.search(r"\bm0\b", t) and i + 2 not in loads]
        assert not others, (name, others)
        total += len(loads)
    assert total > 1000
