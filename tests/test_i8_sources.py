"""What the 8-bit kernels' sources promise the compiler (no GPU needed)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_04052_b200", "csrc")


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if re.search(r"i8|kv8", f) and f.endswith((".cu", ".cuh"))))
def test_operands_are_read_by_ordinary_loads(name):
    """The kernels are resident while the kernel ahead of them, which may have written any of their operands, still runs.  A load that promises memory which does
    not change during the kernel (__ldg, ld.global.nc, a const __restrict__ pointer) may go by a cache that the wait for that kernel does not renew, or move above the wait."""
    with open(os.path.join(CSRC, name)) as f:
        source = re.sub(r"//.*", "", f.read())
    assert not re.search(r"__ldg\s*\(|\.nc\b|__restrict__|__ldca", source), name
