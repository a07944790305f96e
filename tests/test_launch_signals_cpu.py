"""Ordering between kernels and between the CTAs of a cluster, read from the
sources.  A kernel does not let the next one of its stream launch as soon as it
has waited for the one before.  (A kernel that signals at its start and a
cudaStreamWaitEvent between it and the next is the one suspect of a run that
stopped responding.)  Arrivals at another CTA's barrier have cluster scope."""

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


def test_arrivals_at_another_cta_have_cluster_scope():
    """An arrival on a barrier of the cluster without a scope is ordered within its own CTA only."""
    text = open(os.path.join(CSRC, "ff_ptx.cuh")).read()
    arrivals = re.findall(r"mbarrier\.arrive[\w.:]*shared::cluster[\w.:]*", text)
    assert arrivals and all(".cluster.shared::cluster" in a for a in arrivals), arrivals
