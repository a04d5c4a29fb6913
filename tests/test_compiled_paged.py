"""What the compiler made of the paged cache's kernels: the registers hold what they work on."""
import os
import re

from paper_2605_19726_amd import build
from test_compiled_waits import _asm_files  # (builds what is not built)


def test_no_kernel_of_the_paged_cache_spills():
    files = [f for f in _asm_files() if os.path.basename(f).startswith(("attn_decode-", "paged-"))]
    assert len(files) == 2, build.OBJ_DIR
    found, kernels = {}, 0
    for path in files:
        kernel = None
        for line in open(path):
            m = re.match(r"\s*\.amdhsa_(kernel|private_segment_fixed_size) (\S+)", line)
            if m and m.group(1) == "kernel":
                kernel = m.group(2)
                kernels += 1
            elif m and int(m.group(2)):
                found[kernel] = int(m.group(2))
    assert kernels > 20 and found == {}
