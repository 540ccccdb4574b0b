"""How the kernels read global memory."""
import os
import re

import paper_2606_26631_gb300 as prcr

CSRC = os.path.join(os.path.dirname(prcr.__file__), "csrc")


def test_no_read_only_loads():
    """Kernels are launched while the one before them in the stream may still write what they will read, which the read-only path
    (ld.global.nc, __ldg) does not allow: what it reads has to stay as it is as long as the kernel is resident."""
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".cu", ".cuh", ".h")):
            with open(os.path.join(CSRC, name)) as f:
                text = re.sub(r"//[^\n]*", "", f.read())
            assert not re.search(r"global\.nc|__ldg\b|__restrict__", text), name
