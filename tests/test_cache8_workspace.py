"""Workspace sizes of the 8-bit cache's calls, on the host: attention does not pay for the scores of a selection."""
import ctypes

import pytest

import paper_2609_36835_gb300 as pk

OK_BUT_FOR_THE_OUTPUT, WS = 1, 3       # (a missing output is found behind the workspace: nothing is launched)
SIZES = [(64, 8, 131072, 512, 4), (1, 8, 128, 1, 4), (16, 8, 32768, 3, 8), (2, 4, 1 << 20, 100, 1)]


def struct(S, H, cap):
    return pk._Cache8(S, H, cap, 128, *[16] * 10)


def attend(lib, c, n_pos, G, nbytes):
    return lib.arckv_cache_attend(ctypes.byref(c), n_pos, G, 0.0, 16, None, None, 0, None, None, 256, nbytes, 1, None)


def select(lib, c, n_pos, G, nbytes):
    return lib.arckv_cache_select(ctypes.byref(c), n_pos, G, 2, 1, 1, 16, None, None, 256, nbytes, 1, None)


@pytest.mark.parametrize("S,H,cap,n_pos,G", SIZES)
def test_each_call_needs_its_own_share(lib, S, H, cap, n_pos, G):
    c, size = struct(S, H, cap), (S, H, cap, 128, n_pos, G)
    need_attend, need_select = lib.arckv_cache_attend_workspace_bytes(*size), lib.arckv_cache_select_workspace_bytes(*size)
    assert need_select == pk.CACHE_WS_HEADER + 4 * S * H * n_pos * cap // 64
    assert need_attend < 100 << 20                     # partial results of as many CTAs as the GPU has SMs
    assert lib.arckv_cache_workspace_bytes(*size) == max(need_attend, need_select)
    for call, need in ((attend, need_attend), (select, need_select)):
        assert call(lib, c, n_pos, G, need) == OK_BUT_FOR_THE_OUTPUT and call(lib, c, n_pos, G, need - 1) == WS


def test_sizes_that_are_refused_have_no_workspace(lib):
    for bad in ((0, 8, 64, 128, 1, 4), (1, 8, 63, 128, 1, 4), (1, 8, 64, 64, 1, 4), (1, 8, 64, 128, 0, 4)):
        assert lib.arckv_cache_attend_workspace_bytes(*bad) == lib.arckv_cache_select_workspace_bytes(*bad) == 0


def test_calls_without_a_workspace_make_their_own(monkeypatch):
    """A size of zero ends the call before anything is allocated: it tells which one was asked for."""
    asked = []

    class Sizes:
        def __getattr__(self, name):
            return lambda *size: asked.append((name, size)) or 0

    import torch
    monkeypatch.setattr(pk, "load_library", lambda: Sizes())
    monkeypatch.setattr(pk, "status_string", str)
    monkeypatch.setattr(pk, "_on_one_cuda_device", lambda **tensors: None)
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)   # noqa: E731
    c = pk.Cache8(K=z(1, 2, 64, 128, dt=torch.uint8), V=z(1, 2, 64, 128, dt=torch.uint8), k_scale=z(1, 2, 1),
                  v_scale=z(1, 2, 1), bounds=z(1, 2, 1, 2, 128, dt=torch.int8), tail=z(1, 2, 2, 64, 128),
                  tail_amax=z(1, 2, 2, 64), len=z(1, dt=torch.int32), state=z(256, dt=torch.uint8))
    Q = z(1, 2, 3, 4, 128, dt=torch.bfloat16)
    for call in (lambda: pk.cache_attend(c, Q), lambda: pk.cache_select(c, Q, 2), lambda: pk.cache_workspace(c, 3, 4)):
        with pytest.raises(pk.ArckvError):
            call()
    size = (1, 2, 64, 128, 3, 4)
    assert asked == [("arckv_cache_attend_workspace_bytes", size), ("arckv_cache_select_workspace_bytes", size),
                     ("arckv_cache_workspace_bytes", size)]
