"""Waits for what other CTAs of a cluster have sent, in the kernels' sources (no GPU needed).

An asynchronous store to another CTA completes at that CTA's barrier as a release at the cluster's scope.  The wait at the barrier has
to acquire at that scope too: without a scope it is that of the CTA, and reads after it may come before the other CTA's stores.  No run
can show this on a GPU that happens to order them, so the sources are looked at."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1801_00829_b200", "csrc")
SENDERS = [p for p in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))) if "st.async" in open(p).read()]


def test_there_are_such_kernels():
    assert "scan.cuh" in [os.path.basename(p) for p in SENDERS]


@pytest.mark.parametrize("path", SENDERS, ids=os.path.basename)
def test_waits_acquire_at_cluster_scope(path):
    source = open(path).read()
    waits = re.findall(r"mbarrier\.(?:try|test)_wait[\w.:]*", source)
    assert waits and all(".acquire.cluster." in w for w in waits), waits
    # and the cluster's own barrier releases and acquires
    for word in re.findall(r"barrier\.cluster\.(?:arrive|wait)[\w.]*", source):
        assert ".arrive.release" in word or ".wait.acquire" in word, word
