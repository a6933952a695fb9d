"""A rule on the paged cache's kernel sources that no run can show: they start while the kernel before them is still
ending, so memory that it may write must not be loaded as read-only data (which the compiler may move above the wait)."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_36835_gb300" / "csrc"
FILES = sorted(CSRC.glob("pages*.cu*")) + [CSRC / "rotate.cu"]


def code(path):
    text = re.sub(r"/\*.*?\*/", "", path.read_text(), flags=re.S)
    return re.sub(r"//[^\n]*", "", text)


def test_overlapping_kernels_have_no_read_only_loads():
    assert len(FILES) >= 6 and any("launch_pdl(" in code(f) for f in FILES)
    for f in FILES:
        for banned in ("__ldg", "ld.global.nc", "__restrict__"):
            assert banned not in code(f), (f.name, banned)


def test_every_overlapping_kernel_waits_for_the_one_before():
    for f in FILES:
        for body in re.split(r"__global__", code(f))[1:]:
            name = re.search(r"\b(pages_\w+_kernel)\(", body)
            assert name and "pdl_wait();" in body, (f.name, name and name.group(1))
