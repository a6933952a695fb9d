"""What attention over the paged cache could not count: refusals on the host, and a rule on its source."""
import ctypes
import re
from pathlib import Path

import pytest

from paper_2609_36835_gb300 import pages as binding

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_36835_gb300" / "csrc"
SHAPE, WS = 2, 3


def attend(lib, S, H, M, N, G, most):
    """(without a workspace: where the sizes pass, the call ends there)"""
    p = binding._Pages4(S, H, 7, M, 128, 16, 0, 4, 4, 4, 4, 256)
    return lib.arckv_pages_attend(ctypes.byref(p), N, G, most, 0.0, 16, None, 4, 16, None, None, 1 << 40, 1, None)


@pytest.mark.parametrize("S,H,M,N,G,most,code", [
    (1, 8, 1 << 20, 1 << 19, 4, 4096, WS), (64, 8, 1 << 14, 1 << 20, 8, 1 << 16, WS), (1, 1, 46875, 3000000, 8, 3000000, WS),
    (1, 512, 1 << 20, (1 << 17) - 512, 1, 4096, WS), (1, 512, 1 << 20, (1 << 17) - 256, 1, 4096, SHAPE),   # 2^29 (2^9 - 1), 2^38
    (2, 1000, 1 << 20, 1 << 29, 4096, 200, SHAPE)])
def test_a_share_of_all_pages_is_counted_in_31_bits(lib, S, H, M, N, G, most, code):
    assert attend(lib, S, H, M, N, G, most) == code


def test_a_heads_pages_are_counted_in_64_bits():
    """A head has as many steps as its row tiles times its pages, up to 2^40: 2.1 million positions of 8 query heads over as many
    tokens have 2^31.  (Narrowed, a step is negative, and the table is read in front of its beginning.)"""
    body = re.search(r"Segment segment_of\(.*?\n}\n", (CSRC / "pages_tiles.cu").read_text(), re.S).group(0)
    assert re.search(r"long long at = rest - h \* per;", body) and "int at" not in body


@pytest.mark.parametrize("S,H,M", [(4, 8, 128), (1, 1, 1), (4096, 8, 60), (4096, 16, 20000)])
def test_a_workspace_serves_calls_of_fewer_rows(lib, S, H, M):
    """The size never falls as max_count or the query heads of a KV head become more."""
    size = lambda most, G: lib.arckv_pages_attend_workspace_bytes(S, H, M, 128, most, G)
    for G in (1, 2, 3, 4, 8, 9, 16, 33, 128):
        sizes = [size(most, G) for most in list(range(1, 140)) + [255, 256, 257, 1000, 100000]]
        assert sizes[0] > 0 and sizes == sorted(sizes)
    for most in (1, 2, 3, 4, 5, 8, 16, 32, 33, 128, 129):
        sizes = [size(most, G) for G in range(1, 140)]
        assert sizes == sorted(sizes)
