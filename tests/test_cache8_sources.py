"""A rule on the 8-bit cache's kernel sources that no run can show: they start while the kernel before them is still
ending, so memory that it may write must not be loaded as read-only data (which the compiler may move above the wait)."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_36835_gb300" / "csrc"


def code(path):
    text = re.sub(r"/\*.*?\*/", "", path.read_text(), flags=re.S)
    return re.sub(r"//[^\n]*", "", text)


def test_overlapping_kernels_have_no_read_only_loads():
    files = sorted(CSRC.glob("cache8*.cu*"))
    assert len(files) >= 6 and any("launch_pdl(" in code(f) for f in files)
    for f in files:
        for banned in ("__ldg", "ld.global.nc", "__restrict__"):
            assert banned not in code(f), (f.name, banned)


def test_every_overlapping_kernel_waits_for_the_one_before():
    for f in sorted(CSRC.glob("cache8*.cu")):
        text = code(f)
        for body in re.split(r"__global__", text)[1:]:
            name = re.search(r"\b(cache_\w+_kernel)\(", body)
            assert name and "pdl_wait();" in body, (f.name, name and name.group(1))
