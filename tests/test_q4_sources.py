"""Rules that the 4-bit cache's CUDA sources keep and that no run can show."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = {os.path.basename(p): open(p).read()
           for p in sorted(glob.glob(os.path.join(ROOT, "paper_2608_08569_gb300", "csrc", "*q4*.cu*")))}


def test_a_cluster_is_left_by_a_release():
    """A CTA says by a cluster arrive that it is done with the others' shared memory, which may then go: a relaxed
    arrive orders no access before it."""
    arrives = 0
    for f, s in SOURCES.items():
        assert "cluster_arrive_relaxed" not in s and "arrive.relaxed" not in s, f
        arrives += len(re.findall(r"ptx::cluster_arrive\(\)|barrier\.cluster\.arrive\.release", s))
    assert arrives == 3  # pack: one; decode: its start, and what it sends
    ptx = open(os.path.join(ROOT, "paper_2608_08569_gb300", "csrc", "ptx.cuh")).read()
    assert "barrier.cluster.arrive.release.aligned" in ptx
