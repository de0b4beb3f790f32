"""What the kernels' sources must not hold."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_20289_gb300", "csrc")
FILES = sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh")))


@pytest.mark.parametrize("name", FILES)
def test_copies_name_no_other_cta(name):
    """A bulk copy fills the shared memory of the CTA that asks for it alone: no multicast.  The operators'
    workspaces are the caller's, and every replica of a job on several GPUs runs these kernels."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    for instruction in re.findall(r"cp\.async\.bulk[^\s\"]*", text):
        assert "multicast" not in instruction, instruction
