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


@pytest.mark.parametrize("code,S,rows", [(2, 3, True), (1, 3, True), (7, 3, False), (2, 5000, False)])
def test_an_error_found_by_the_extensions_kernel_has_its_rows(lib, monkeypatch, code, S, rows):
    """(the library is a stand-in but for its sizes; 5000 requests it refuses before it runs)"""
    import types

    import torch

    import paper_2609_36835_gb300 as pk
    real = pk.load_library()
    stand_in = types.SimpleNamespace(arckv_pages_extend=lambda *args: code, arckv_status_string=real.arckv_status_string,
                                     arckv_pages_attend_workspace_bytes=real.arckv_pages_attend_workspace_bytes)
    monkeypatch.setattr(pk, "load_library", lambda: stand_in)
    monkeypatch.setattr(pk, "_on_one_cuda_device", lambda **tensors: None)
    monkeypatch.setattr(pk, "_current_handle", lambda device: 11)
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 1)
    room = torch.zeros(1024, dtype=torch.uint8)
    state = room[-room.data_ptr() % 256:][:256]
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    p = pk.Pages4(data=torch.zeros(4, 2, pk.PAGE_BYTES, dtype=torch.uint8), table=i32(S, 4), len=i32(S), free=i32(4), n_free=i32(1), state=state)
    with pytest.raises(pk.ArckvError) as e:
        pk.pages_extend(p, i32(S), 7)
    assert e.value.code == code and (e.value.rows is not None) == rows
    if rows:
        assert [len(x) for x in e.value.rows] == [S + 1, 7, 7]
