"""What attention over the 8-bit cache could not count: refusals on the host, and a rule on its source."""
import ctypes
import re
from pathlib import Path

import pytest

import paper_2609_36835_gb300 as pk

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_36835_gb300" / "csrc"
BAD, SHAPE = 1, 2


@pytest.mark.parametrize("H,cap,n_pos,G,code", [
    (1, 1 << 22, 2100000, 8, BAD), (8, 1 << 17, 1 << 17, 8, BAD), (1, 1 << 26, 1 << 24, 3, BAD),      # 2^20 (3 * 2^16 + 1)
    (1, 1 << 26, 1 << 24, 4, SHAPE), (2, 1 << 26, 1 << 24, 32, SHAPE)])
def test_a_share_of_all_blocks_is_counted_in_31_bits(lib, H, cap, n_pos, G, code):
    """(the negative scale ends a call whose sizes pass)"""
    c = pk._Cache8(1, H, cap, 128, *[16] * 10)
    assert lib.arckv_cache_attend(ctypes.byref(c), n_pos, G, -1.0, 16, None, None, 0, 16, None, 256, 1 << 40, 1, None) == code


def test_a_heads_blocks_are_counted_in_64_bits():
    """A head has as many steps as its row tiles times its blocks, 2^31 for 2.1 million positions of 8 query heads over as many
    tokens.  (Narrowed, a step is negative, and keys in front of the head's are read.)"""
    body = re.search(r"Segment segment_of\(.*?\n}\n", (CSRC / "cache8_tiles.cu").read_text(), re.S).group(0)
    assert re.search(r"long long at = rest - h \* per;", body) and "int at" not in body
