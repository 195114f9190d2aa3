"""Loads that take memory to be constant while a kernel runs, in sources whose kernels
may start before the kernel in front of them has ended.

``ee_prompt_slots`` writes block tables, lengths and offsets; the kernels that read
them start early (programmatic dependent launch) and wait for it on the device.  A
non-coherent load needs data that nobody writes during the reader's whole lifetime,
so none of these may use one.  What ``match.cu`` and the weights' rearrangement in
``lmhead.cu`` read so (code tokens, weights) is the caller's, and no kernel of the
library writes it."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_02780_gb300", "csrc")
CALLERS_ONLY = {"match.cu": 2, "lmhead.cu": 2}


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu*"))), ids=os.path.basename)
def test_no_noncoherent_load_of_what_a_kernel_writes(path):
    with open(path) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    found = re.findall(r"ld\.global\.nc|\b__ldg\s*\(|\b__restrict__\b", code)
    assert len(found) == CALLERS_ONLY.get(os.path.basename(path), 0), found
