"""Layer norm's backward kernels live in registers: one that spills pays for
every spilled number in each row (a form of 16 waves and 3 vectors a lane took
260 us for 2000 rows of 21504, the streaming form 100).  Checked on the built
library."""

import os
import re
import subprocess

import paper_2609_02846_amd as ue
from paper_2609_02846_amd import build as ue_build
from test_mfma_wait import LLVM, _code_objects


def test_backward_kernels_use_no_scratch(tmp_path):
    if not os.path.exists(ue.LIB_PATH):
        ue_build.build(verbose=False)
    found, spilling = 0, set()
    for i, obj in enumerate(_code_objects(ue.LIB_PATH)):
        if b"norm_bwd_kernel" not in obj:
            continue
        f = tmp_path / f"{i}.o"
        f.write_bytes(obj)
        name = None
        for line in subprocess.run([f"{LLVM}/llvm-objdump", "-d", str(f)], capture_output=True, text=True,
                                   check=True).stdout.splitlines():
            m = re.match(r"[0-9a-f]+ <(.+)>:$", line)
            if m:
                name = m.group(1)
                found += "norm_bwd" in name
            elif "scratch_" in line and "norm_bwd" in name:
                spilling.add(name)
    assert found > 20 and not spilling, sorted(spilling)
