"""What the kernels of the student-body operators may not contain, whatever the tests on a GPU happen to see."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_03796_b200", "csrc")
EARLY = ["act8.cuh", "act8_dweight.cuh", "block_norm_kernels.cuh", "gated_kernels.cuh"]


def _code(name):
    """A source file without its comments."""
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"/\*.*?\*/", "", re.sub(r"//[^\n]*", "", f.read()), flags=re.S)


@pytest.mark.parametrize("name", EARLY)
def test_kernels_that_start_early_read_coherently(name):
    """These kernels start while the one before them on the stream still writes their inputs, and read them after
    griddepcontrol.wait. The non-coherent path (ld.global.nc, __ldg, and what the compiler makes of a const __restrict__
    parameter) is defined only for memory that is read-only for a kernel's whole lifetime: a line of the call before may
    be returned. The case that shows it most plainly is a weight gradient that reads the old value of the buffer that it
    overwrites."""
    code = _code(name)
    assert "grid_dependency_wait" in code
    assert not re.search(r"\.nc\b", code) and "__ldg" not in code
    for declaration in re.findall(r"[^,;(){}]*__restrict__", code):
        assert "const" not in declaration, declaration


def test_the_pairs_leader_acquires_what_the_peer_wrote():
    """The leader's MMAs read the peer CTA's shared memory and overwrite its tensor memory: what tells the leader that it
    may has to be released and acquired for the cluster. An arrival's and a wait's default scope is the CTA."""
    code = _code("act8_dweight.cuh")
    assert "mbar_arrive_cluster(" not in code
    for barrier in ("full", "tempty"):
        assert f"mbar_wait<true>({barrier}(" in code and f"mbar_wait({barrier}(" not in code
        assert f"mbar_arrive_pair(map_to_cta({barrier}(" in code
    prims = _code("sm100_prims.cuh")
    for part in ("fence.release.sync_restrict::shared::cta.cluster", "mbarrier.arrive.relaxed.cluster",
                 "mbarrier.try_wait.parity.relaxed.cluster", "fence.acquire.sync_restrict::shared::cluster.cluster"):
        assert part in prims
