"""The TMEM instructions with .sync.aligned want all lanes of a warp at them together.  Each stands in a function of its own,
which brings the lanes back together itself: what its callers did before (single lanes that arrive at a barrier, stores of
the lanes whose row or column is there) does not count then.  The two waits follow the loads and stores that they wait for."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_08991_gb300", "csrc")
ACCESS = re.compile(r"tcgen05\.(?:ld|st|alloc|dealloc|relinquish_alloc_permit)\.[a-z0-9_:.]*sync\.aligned")


def _accesses():
    """(file, instruction, the enclosing function's text before it)."""
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        for m in ACCESS.finditer(text):
            yield name, m.group(0), text[text.rindex("__device__ __forceinline__", 0, m.start()):m.start()]


def test_every_access_brings_its_warp_together():
    found = list(_accesses())
    assert {n for n, _, _ in found} >= {"tc_common.cuh", "q4.cu"} and len(found) >= 5
    for name, access, before in found:
        assert before.count("\n}\n") == 0, (name, access)          # the function that the access stands in
        if "relinquish" in access:
            continue                                               # (directly behind an allocation)
        assert "__syncwarp();" in before, (name, access)


def test_barriers_of_some_warps_bring_them_together():
    """bar.sync with a number of threads is aligned, too."""
    with open(os.path.join(CSRC, "common.cuh")) as f:
        text = f.read()
    body = text[text.index("void named_barrier("):]
    body = body[:body.index("\n}")]
    assert body.index("__syncwarp();") < body.index("bar.sync")
