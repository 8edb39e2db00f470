"""What a kernel asks of a device is asked of each device (no GPU): the calls without a handle
may come from any of a process's devices, and a flag of the process would serve the first."""
import glob
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2608_28099_gb300", "csrc")
NO_HANDLE = sorted(os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "sp_cache*.cu")) +
                   glob.glob(os.path.join(CSRC, "sp_tree_*.cu")))


@pytest.mark.parametrize("name", NO_HANDLE)
def test_no_flag_of_the_process(name):
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"\bstatic\s+(?:bool|int)\s+\w+\s*=", text)
    assert "cudaFuncSetAttribute" not in text  # allow_smem, by device
    for table in re.findall(r"\bstatic\s+(?:bool|int)\s+\w+\[(\w+)\]", text):
        assert table == "MAX_DEVICES"
