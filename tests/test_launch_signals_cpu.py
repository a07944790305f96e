"""Where kernels let the next one of their stream launch, read from the
sources: never as soon as they have waited for the one before.  (A kernel that
signals at its start and a cudaStreamWaitEvent between it and the next is the
one suspect of a run that stopped responding.)"""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_08573_gb300", "csrc")


def test_no_kernel_signals_before_its_work():
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"griddep_wait\(\);", text):
            found += 1
            assert not re.match(r"\s*(ptx::)?griddep_launch_dependents", text[m.end():]), os.path.basename(path)
    assert found > 10
