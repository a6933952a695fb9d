"""What the 8-bit cache's Python calls do around the library call, on the host: the library is a stand-in that records
its calls, and tensors that record the streams they are used on take the place of device memory."""
import contextlib
import types

import pytest
import torch

import paper_2609_36835_gb300 as pk

S, H, CAP, G = 2, 3, 128, 4


class Recorded(torch.Tensor):
    """A host tensor that notes the streams it is recorded on."""
    used = None

    def record_stream(self, stream):
        self.used.append((self.data_ptr(), stream))


class Stream:
    cuda_stream = 77


@pytest.fixture
def rig(monkeypatch):
    """The cache calls over a stand-in library; `calls` are its calls, `used` the recorded (address, stream)."""
    r = types.SimpleNamespace(calls=[], used=[], guards=[], device=0, devices=2)
    monkeypatch.setattr(Recorded, "used", r.used)

    def entry(name, value=0):
        def call(*args):
            r.calls.append((name, args, list(r.guards)))
            return value
        return call

    lib = types.SimpleNamespace(**{n: entry(n) for n in ("arckv_cache_append", "arckv_cache_read", "arckv_cache_attend",
                                                         "arckv_cache_select", "arckv_query_status")},
                                arckv_cache_workspace_bytes=entry("arckv_cache_workspace_bytes", 8192))
    monkeypatch.setattr(pk, "load_library", lambda: lib)
    monkeypatch.setattr(pk, "_on_one_cuda_device", lambda **tensors: None)
    monkeypatch.setattr(pk, "_current_handle", lambda device: 11)

    @contextlib.contextmanager
    def guard(what):
        r.guards.append(what)
        yield
        r.guards.pop()

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: object())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: r.device)
    monkeypatch.setattr(torch.cuda, "device_count", lambda: r.devices)
    monkeypatch.setattr(torch.cuda, "stream", guard)
    monkeypatch.setattr(torch.cuda, "device", guard)
    return r


def z(*shape, dt=torch.float32):
    return torch.zeros(*shape, dtype=dt).as_subclass(Recorded)


def cache(bias=True):
    nb = CAP // 64
    return pk.Cache8(K=z(S, H, CAP, 128, dt=torch.uint8), V=z(S, H, CAP, 128, dt=torch.uint8), k_scale=z(S, H, nb),
                     v_scale=z(S, H, nb), bounds=z(S, H, nb, 2, 128, dt=torch.int8), tail=z(S, H, 2, 64, 128),
                     tail_amax=z(S, H, 2, 64), len=z(S, dt=torch.int32), bias=z(S, H, CAP) if bias else None,
                     state=z(256, dt=torch.uint8))


ARRAYS = ("K", "V", "k_scale", "v_scale", "bounds", "tail", "tail_amax", "len", "state")


def arguments(n=5):
    return dict(rows=z(S, H, n, 128, dt=torch.bfloat16), more=z(S, H, n, 128, dt=torch.bfloat16), bias=z(S, H, n),
                at=z(S, dt=torch.int32), counts=z(S, dt=torch.int32), Q=z(S, H, 2, G, 128, dt=torch.bfloat16),
                blocks=z(S, H, 2, 3, dt=torch.int32), out=z(S, H, 2, G, 128), ws=z(8192, dt=torch.uint8))


CALLS = {
    "append": (("rows", "more", "bias", "at", "counts"),
               lambda c, a, **kw: pk.cache_append(c, a["rows"], a["more"], bias=a["bias"], at=a["at"], counts=a["counts"],
                                                  **kw)),
    "read": ((), lambda c, a, **kw: pk.cache_read(c, 0, 4, **kw)),
    "attend": (("Q", "blocks", "out", "ws"),
               lambda c, a, **kw: pk.cache_attend(c, a["Q"], blocks=a["blocks"], out=a["out"], ws=a["ws"], **kw)),
    "select": (("Q", "ws"), lambda c, a, **kw: pk.cache_select(c, a["Q"], 3, ws=a["ws"], **kw)),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("bias", [True, False])
def test_every_tensor_is_recorded_on_another_stream(rig, name, bias):
    """All memory that a call reads or writes on a stream other than the current one: the cache's arrays too."""
    c, a, stream = cache(bias=bias or name == "append"), arguments(), Stream()
    given, call = CALLS[name]
    call(c, a, stream=stream, check=False)
    assert [n for n, _, _ in rig.calls] == ["arckv_cache_" + name]
    want = {getattr(c, n).data_ptr() for n in ARRAYS} | {a[n].data_ptr() for n in given}
    if c.bias is not None:
        want.add(c.bias.data_ptr())
    assert {address for address, _ in rig.used} == want
    assert all(s is stream for _, s in rig.used)


@pytest.mark.parametrize("name", CALLS)
def test_nothing_is_recorded_on_the_current_stream(rig, name):
    CALLS[name][1](cache(), arguments(), check=False)
    assert not rig.used


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("check", [True, False])
def test_the_library_runs_with_the_caches_device_current(rig, name, check):
    """A cache on another device than the current one: the call is made inside a guard for the cache's device."""
    c = cache()
    rig.device = 1                       # (host tensors: a device without an index, which no current device equals)
    CALLS[name][1](c, arguments(), check=check)
    (entry, args, guards), = rig.calls
    assert entry == "arckv_cache_" + name and guards == [c.K.device] and not rig.guards
    assert args[-1] == 11                # the current stream of that device


def test_no_guard_where_the_device_is_current(rig):
    c = cache()
    rig.device = c.K.device.index
    for name in CALLS:
        CALLS[name][1](c, arguments())
    assert len(rig.calls) == len(CALLS) and not any(guards for _, _, guards in rig.calls)


def test_no_guard_where_there_is_one_device(rig):
    rig.devices, rig.device = 1, 1
    c = cache()
    for name in CALLS:
        CALLS[name][1](c, arguments())
    assert len(rig.calls) == len(CALLS) and not any(guards for _, _, guards in rig.calls)


def test_the_status_is_read_on_the_words_device(rig):
    word = types.SimpleNamespace(device=torch.device("cuda", 1), is_contiguous=lambda: True, data_ptr=lambda: 4096)
    assert pk.arckv_query_status(word) == 0
    assert rig.calls == [("arckv_query_status", (4096, 11), [word.device])]
    rig.device = 1
    assert pk.arckv_query_status(word) == 0 and rig.calls[1][2] == []
    assert pk.arckv_query_status(4096, stream=Stream()) == 0 and rig.calls[2][1] == (4096, 77)


@pytest.mark.parametrize("name", ["attend", "select"])
@pytest.mark.parametrize("ws", [torch.zeros(8192, dtype=torch.uint8, device="meta"), torch.zeros(8192, dtype=torch.int8),
                                torch.zeros(4096), torch.zeros(16384, dtype=torch.uint8)[::2], 4096])
def test_workspaces_that_are_not_bytes_on_the_device_are_refused(rig, name, ws):
    """Another device or type, gaps, or an address: the library would take the numbers as they are."""
    with pytest.raises(ValueError, match="ws"):
        CALLS[name][1](cache(), {**arguments(), "ws": ws})
    assert not rig.calls


def test_a_list_without_entries_is_refused(rig):
    """The address of an empty tensor is null, which stands for no list: every block would be read."""
    with pytest.raises(ValueError, match="blocks"):
        CALLS["attend"][1](cache(), {**arguments(), "blocks": z(S, H, 2, 0, dt=torch.int32)})
    assert not rig.calls


@pytest.mark.parametrize("m,last,first", [(1, 1, 0), (1, 0, 1), (2, 1, 1), (2, 2, 0), (9, 1, 1)])
def test_the_first_block_is_kept_where_there_is_room(rig, m, last, first):
    c, a = cache(), arguments()
    pk.cache_select(c, a["Q"], m, keep_last=last, ws=a["ws"])
    pk.cache_select(c, a["Q"], m, keep_first=2, keep_last=last, ws=a["ws"])
    assert [args[3:6] for _, args, _ in rig.calls] == [(m, first, last), (m, 2, last)]


def test_outputs_whose_rows_share_memory_are_refused(rig):
    c, a = cache(), arguments()
    whole = torch.zeros(S, 2, H, G, 128)
    for out in (torch.zeros(S, 1, 2, G, 128).expand(S, H, 2, G, 128), torch.zeros(1, H, 2, G, 128).expand(S, H, 2, G, 128),
                torch.zeros(9999).as_strided((S, H, 2, G, 128), (3 * H * 512, 2 * 512, 512 - 128, 128, 1))):
        with pytest.raises(ValueError, match="out"):
            CALLS["attend"][1](c, {**a, "out": out})
    assert not rig.calls
    for out in (whole.transpose(1, 2), torch.zeros(S, H, 5, G, 128)[:, :, 1:3], torch.zeros(2 * S, H, 4, G, 128)[::2, :, ::2],
                torch.zeros(H, S, 2, G, 128).transpose(0, 1)):
        CALLS["attend"][1](c, {**a, "out": out})
    assert len(rig.calls) == 4


@pytest.mark.parametrize("beyond", [1 << 32, -(1 << 32), 1 << 31])
def test_numbers_past_32_bits_are_refused(rig, beyond):
    """The library takes 32-bit integers: token 2^32 would be read as token 0."""
    c, a = cache(), arguments()
    for call in (lambda: pk.cache_read(c, beyond, 4), lambda: pk.cache_select(c, a["Q"], 3, keep_first=beyond, ws=a["ws"]),
                 lambda: pk.cache_select(c, a["Q"], 3, keep_last=beyond, ws=a["ws"])):
        with pytest.raises(ValueError, match="out of range"):
            call()
    assert not rig.calls
