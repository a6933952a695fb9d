"""What the paged cache's and the rotation's Python calls do around the library call, on the host: the library is a stand-in
that records its calls, and tensors that record the streams they are used on take the place of device memory."""
import contextlib
import types

import pytest
import torch

import paper_2609_36835_gb300 as pk

S, H, P, M, G, N = 2, 3, 7, 4, 4, 5


class Recorded(torch.Tensor):
    """A host tensor that notes the streams it is recorded on and calls itself a CUDA tensor where asked."""
    used = None

    def record_stream(self, stream):
        self.used.append((self.data_ptr(), stream))


class Stream:
    cuda_stream = 77


@pytest.fixture
def rig(monkeypatch):
    r = types.SimpleNamespace(calls=[], used=[], guards=[], device=0, devices=2)
    monkeypatch.setattr(Recorded, "used", r.used)

    def entry(name, value=0):
        def call(*args):
            r.calls.append((name, args, list(r.guards)))
            return value
        return call

    lib = types.SimpleNamespace(arckv_status_string=lambda code: b"an error", **{n: entry(n) for n in ("arckv_pages_extend", "arckv_pages_truncate", "arckv_pages_append",
                                                         "arckv_pages_read", "arckv_pages_attend", "arckv_query_status")},
                                arckv_pages_attend_workspace_bytes=entry("arckv_pages_attend_workspace_bytes", 8192))
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


def i32(*shape):
    return z(*shape, dt=torch.int32)


def pages(bias=True):
    return pk.Pages4(data=z(P, H, pk.PAGE_BYTES, dt=torch.uint8), table=i32(S, M), len=i32(S), free=i32(P), n_free=i32(1),
                     bias=z(P, H, 64) if bias else None, state=z(256, dt=torch.uint8))


ARRAYS = ("data", "table", "len", "free", "n_free", "state")


def arguments():
    return dict(counts=i32(S), lens=i32(S), rows=z(N, H, 128, dt=torch.bfloat16), more=z(N, H, 128, dt=torch.bfloat16), bias=z(N, H),
                slots=i32(N), Q=z(N, H, G, 128, dt=torch.bfloat16), starts=i32(S + 1), out=z(N, H, G, 128, dt=torch.bfloat16),
                ws=z(8192, dt=torch.uint8))


CALLS = {
    "extend": (("counts",), lambda p, a, **kw: pk.pages_extend(p, a["counts"], N, **kw)),
    "truncate": (("lens",), lambda p, a, **kw: pk.pages_truncate(p, a["lens"], **kw)),
    "append": (("rows", "more", "slots", "bias"),
               lambda p, a, **kw: pk.pages_append(p, a["rows"], a["more"], a["slots"], bias=a["bias"], **kw)),
    "read": (("slots",), lambda p, a, **kw: pk.pages_read(p, a["slots"], **kw)),
    "attend": (("Q", "starts", "out", "ws"),
               lambda p, a, **kw: pk.pages_attend(p, a["Q"], a["starts"], out=a["out"], ws=a["ws"], **kw)),
}


@pytest.mark.parametrize("name", CALLS)
def test_every_tensor_is_recorded_on_another_stream(rig, name):
    p, a, stream = pages(), arguments(), Stream()
    given, call = CALLS[name]
    call(p, a, stream=stream, check=False)
    assert [n for n, _, _ in rig.calls] == ["arckv_pages_" + name]
    want = {getattr(p, n).data_ptr() for n in ARRAYS + ("bias",)} | {a[n].data_ptr() for n in given}
    assert {address for address, _ in rig.used} == want and all(s is stream for _, s in rig.used)


@pytest.mark.parametrize("name", CALLS)
def test_nothing_is_recorded_on_the_current_stream(rig, name):
    CALLS[name][1](pages(), arguments(), check=False)
    assert not rig.used


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("check", [True, False])
def test_the_library_runs_with_the_pages_device_current(rig, name, check):
    p = pages()
    rig.device = 1                       # (host tensors: a device without an index, which no current device equals)
    CALLS[name][1](p, arguments(), check=check)
    (entry, args, guards), = rig.calls
    assert entry == "arckv_pages_" + name and guards == [p.data.device] and not rig.guards


@pytest.mark.parametrize("name", CALLS)
def test_an_error_is_raised(rig, name):
    setattr(pk.load_library(), "arckv_pages_" + name, lambda *args: 2)
    with pytest.raises(pk.ArckvError):
        CALLS[name][1](pages(), arguments())


def test_calls_without_rows_make_no_call(rig):
    p, none = pages(), lambda *s, dt=torch.bfloat16: torch.zeros(0, *s, dtype=dt)
    pk.pages_append(p, none(H, 128), none(H, 128), none(dt=torch.int32))
    K, V = pk.pages_read(p, none(dt=torch.int32))
    O = pk.pages_attend(p, none(H, G, 128), i32(S + 1), ws=arguments()["ws"])
    assert K.shape == V.shape == (0, H, 128) and O.shape == (0, H, G, 128) and not rig.calls


@pytest.mark.parametrize("name,change", [
    ("extend", dict(counts=i32(S + 1))), ("extend", dict(counts=z(S))), ("extend", dict(counts=torch.zeros(2 * S, dtype=torch.int32)[::2])),
    ("extend", dict(counts=[0, 1])), ("truncate", dict(lens=i32(S, 1))),
    ("append", dict(rows=z(N, H, 64))), ("append", dict(rows=z(N, H, 128))), ("append", dict(rows=z(N, H + 1, 128, dt=torch.bfloat16))),
    ("append", dict(rows=z(N, H, 256, dt=torch.bfloat16)[..., ::2])), ("append", dict(slots=i32(N + 1))),
    ("append", dict(slots=z(N, dt=torch.int64))), ("append", dict(bias=z(N, H + 1))), ("append", dict(bias=z(N, H, dt=torch.bfloat16))),
    ("read", dict(slots=i32(N, 1))), ("attend", dict(Q=z(N, H, G, 64, dt=torch.bfloat16))), ("attend", dict(Q=z(N, H, G, 128))),
    ("attend", dict(Q=z(N, H, 2 * G, 128, dt=torch.bfloat16)[:, :, ::2])), ("attend", dict(starts=i32(S))),
    ("attend", dict(out=z(N, H, G, 128))), ("attend", dict(out=z(1, H, G, 128, dt=torch.bfloat16).expand(N, H, G, 128))),
    ("attend", dict(ws=z(8192))), ("attend", dict(ws=8192))])
def test_refusals(rig, name, change):
    with pytest.raises(ValueError):
        CALLS[name][1](pages(), {**arguments(), **change})
    assert not rig.calls


@pytest.mark.parametrize("call", [lambda p: pk.pages_extend(p, i32(S), -1), lambda p: pk.pages_extend(p, i32(S), 1 << 30),
                                  lambda p: pk.pages_workspace(p, 1 << 31, 4), lambda p: pk.pages_read(p, i32(N), dtype=torch.float16),
                                  lambda p: pk.pages_attend(p, arguments()["Q"], i32(S + 1), max_count=1 << 40)])
def test_numbers_past_the_librarys_range_are_refused(rig, call):
    with pytest.raises(ValueError):
        call(pages())
    assert not rig.calls


def test_a_bias_needs_pages_that_hold_one(rig):
    a = arguments()
    with pytest.raises(ValueError):
        pk.pages_append(pages(bias=False), a["rows"], a["more"], a["slots"], bias=a["bias"])


@pytest.mark.parametrize("change", [dict(data=z(P, H, 100, dt=torch.uint8)), dict(table=z(S, M)), dict(len=i32(S + 1)), dict(free=i32(P + 1)),
                                    dict(n_free=i32(2)), dict(bias=z(P, H, 32)), dict(state=z(128, dt=torch.uint8))])
def test_pages_of_other_shapes_are_refused(rig, change):
    p = pages()
    with pytest.raises(ValueError):
        pk.Pages4(**{**{n: getattr(p, n) for n in ARRAYS + ("bias",)}, **change})


def test_a_rotation_refuses_host_tensors():
    r = pk.rotary(64, device="cpu")
    with pytest.raises(ValueError):
        pk.rotate(r, torch.zeros(3, dtype=torch.int32), torch.zeros(3, 2, 128))


def test_strided_rows_reach_the_library(rig):
    p, a = pages(), arguments()
    fused = z(N, 3 * H, 128, dt=torch.bfloat16)
    pk.pages_append(p, fused[:, :H], fused[:, H:2 * H], a["slots"], check=False)
    args = rig.calls[0][1]
    assert list(args[3]) == [3 * H * 128, 128] and list(args[5]) == [3 * H * 128, 128]
    assert args[4] - args[2] == H * 128 * 2
