"""What the compiler does not check in the kernels' sources (no GPU needed)."""
from __future__ import annotations

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2403_10616_b200", "csrc")


def test_dynamic_shared_memory_is_declared_at_16_bytes():
    """Vectors of 16 bytes are read from it, and without a declared alignment it begins wherever the kernel's
    static shared memory ends.  Buffers of plain bytes are aligned by their kernels before use."""
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        for line in re.findall(r"extern\s+__shared__[^;]*;", open(path).read()):
            found += 1
            declared = re.search(r"__align__\((\d+)\)", line)
            bytes_only = re.search(r"\b(uint8_t|unsigned char)\s+\w+\[\]", line)
            assert bytes_only or (declared and int(declared.group(1)) % 16 == 0), (os.path.basename(path), line)
    assert found >= 5
