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


def test_every_kernel_checks_its_rows_in_the_checked_build():
    """VOXZIP_IN_RANGE stands in each kernel of the 4-bit cache, so that the checked build's runs show what they touch."""
    kernels = [(f, m.group(1), m.start()) for f, s in SOURCES.items() for m in re.finditer(r"__global__[^;{]*?(\w+)\(const \w+ p\)", s)]
    assert sorted(k for _, k, _ in kernels) == ["decode_q4_mma_kernel", "decode_q4_rows_kernel", "evict_q4_kernel", "q4_pack_kernel",
                                                "q4_unpack_kernel"]
    for f, k, at in kernels:
        s = SOURCES[f]
        end = min([a for g, _, a in kernels if g == f and a > at] + [s.find("cudaError_t", at)])
        assert s.count("VOXZIP_IN_RANGE", at, end) >= 1, k
