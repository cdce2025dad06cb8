"""Rules that the kernels' sources keep.  No GPU."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2209_13258_b200", "csrc")


def test_nothing_is_read_through_the_read_only_path():
    """Every kernel starts while the one before it on the stream still runs, and may read what that one writes: loads of
    data that must not change during the kernel (__ldg, ld.global.nc, pointers to const that are __restrict__) are not
    allowed to see it."""
    files = [f for f in glob.glob(os.path.join(CSRC, "*")) if f.endswith((".cu", ".cuh", ".h"))]
    assert len(files) > 5
    for f in files:
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(f).read(), flags=re.S)
        for word in (r"__ldg\w*", r"ld\.global\.(\w+[.:]*)*nc\b", r"__restrict__"):
            assert not re.search(word, code), (os.path.basename(f), word)


def test_every_kernel_that_overlaps_waits_before_it_reads():
    """griddepcontrol.wait in every kernel that lets the next one start early, or is launched that way."""
    for f in glob.glob(os.path.join(CSRC, "*.cu*")):
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(f).read(), flags=re.S)
        starts = [m.start() for m in re.finditer(r"__global__ ", code)] + [len(code)]
        for a, b in zip(starts, starts[1:]):
            body = code[a:b]
            if "pdl_launch_dependents()" in body or "griddepcontrol.launch_dependents" in body:
                assert "pdl_wait()" in body or "griddepcontrol.wait" in body, (os.path.basename(f), body[:120])
