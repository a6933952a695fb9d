"""Index and bias arrays off the 4-byte grid are refused on the host by the 8-bit cache's entries: a kernel that loaded
from them would fault.  (Each call here is refused before anything is launched: where the arrays are aligned, a missing
argument behind them is found.)"""
import ctypes

import pytest

import paper_2609_36835_gb300 as pk

BAD, SHAPE = 1, 2


def struct(bias):
    return pk._Cache8(2, 3, 128, 128, *([16] * 5 + [bias] + [16] * 4))


def test_the_struct_is_as_expected():
    assert [n for n, _ in pk._Cache8._fields_[4:]].index("bias") == 5


@pytest.mark.parametrize("name", ["bias", "at", "counts"])
@pytest.mark.parametrize("address", [18, 17, 19])
def test_append(lib, name, address):
    given = {"bias": None, "at": None, "counts": None, name: address}
    code = lib.arckv_cache_append(ctypes.byref(struct(16)), 4, 16, None, 16, None, given["bias"], given["at"],
                                  given["counts"], 1, None)
    assert code == BAD


@pytest.mark.parametrize("address", [18, 17, 19])
def test_attend(lib, address):
    # m = 0 is refused as a shape behind the pointers
    args = lambda blocks: (ctypes.byref(struct(0)), 1, 4, 0.0, 16, None, blocks, 0, 16, None, 256, 1 << 40, 1, None)
    assert lib.arckv_cache_attend(*args(address)) == BAD
    assert lib.arckv_cache_attend(*args(16)) == lib.arckv_cache_attend(*args(20)) == SHAPE
