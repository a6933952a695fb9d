"""The paged 4-bit cache and rotary positions without a GPU: their plain form on cases worked out by hand, frequencies,
workspace sizes and refusals on the host."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import pages4 as ref
import paper_2609_36835_gb300 as pk
from paper_2609_36835_gb300 import pages as binding

BAD, SHAPE, WS, UNSUPPORTED = 1, 2, 3, 8


# ------------------------------------------------------------------ plain form

def test_codes_by_hand():
    x = np.zeros((1, 128), np.float32)
    x[0, :32] = np.arange(32) / 31 * 15 - 3          # range 15 from -3: scale 1
    got = ref.held(x, 32)
    assert np.array_equal(got[0, :32], np.rint(np.arange(32) / 31 * 15) - 3)
    assert not got[0, 32:].any()                     # zeros are held exactly
    half = np.array([[0.0, 15.0] + [2.5, 3.5] * 63], np.float32)
    assert set(ref.held(half, 128)[0]) == {0.0, 15.0, 2.0, 4.0}      # halves go to the even code


def test_values_are_within_half_a_step_and_the_scales_roundings():
    x = np.random.default_rng(0).normal(size=(50, 128)).astype(np.float32)
    for group in (32, 128):
        y = x.reshape(50, -1, group)
        span = (y.max(-1) - y.min(-1))[..., None].astype(np.float64)
        size = np.abs(y).max(-1)[..., None]
        # half a step, what m and s lose to bf16 (2^-9 of each: at the far end 15 s and m), with a tenth to spare
        assert np.all(np.abs(ref.held(x, group).reshape(y.shape) - y) <= span / 30 + 1.1 * 2.0 ** -8 * (span + size))


def test_bf16_rounding_is_torchs():
    x = np.random.default_rng(1).normal(size=4096).astype(np.float32) * np.float32(2.0) ** np.arange(-20, 20).repeat(103)[:4096].astype(np.float32)
    assert np.array_equal(ref.as_bf16(x), torch.from_numpy(x).to(torch.bfloat16).float().numpy())


def test_tables_by_hand():
    t = ref.Tables(3, 4, 5)
    starts, slots, pos = t.extend([65, 0, 2], 70)
    assert starts.tolist() == [0, 65, 65, 67] and t.len.tolist() == [65, 0, 2]
    assert t.table[0, :2].tolist() == [0, 1] and t.table[2, 0] == 2
    assert slots[64] == 64 and slots[66] == 2 * 64 + 1 and slots[67] == -1 and pos[64] == 64 and pos[69] == -1
    before = (t.table.copy(), t.len.copy(), list(t.free))
    t.extend([63, 64, 63], 190)
    assert t.len.tolist() == [128, 64, 65] and len(t.free) == 0
    t.truncate([65, 0, 2])
    assert np.array_equal(t.table, before[0]) and np.array_equal(t.len, before[1]) and t.free == before[2]
    t.extend([64, 129, 62], 1000)                    # two pages left: the first takes one, the second needs three; 62 fit
    assert t.len.tolist() == [129, 0, 64]


def test_rotation_by_hand():
    x = np.zeros((1, 1, 16))
    x[0, 0, 0], x[0, 0, 8] = 1.0, 0.0
    quarter = [2 ** 62] + [0] * 7
    assert np.allclose(ref.rotate(x, [1], quarter)[0, 0, [0, 8]], [0, 1])
    assert np.allclose(ref.rotate(x, [5], quarter, transpose=True)[0, 0, [0, 8]], [0, -1])
    assert np.allclose(ref.rotate(x, [2], quarter, interleaved=True)[0, 0, [0, 1]], [-1, 0])
    assert np.allclose(ref.rotate(x, [-1], quarter), x)


# ----------------------------------------------------------------- frequencies

def test_frequencies_by_hand():
    f, factor = pk.rotary_frequencies(8, 10000.0)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001]) and factor == 1.0
    assert np.allclose(pk.rotary_frequencies(8, 10000.0, {"kind": "linear", "factor": 4})[0], np.array(f) / 4)
    g, _ = pk.rotary_frequencies(8, 10000.0, {"kind": "base", "factor": 8})
    assert g[0] == 1.0 and np.isclose(g[3], f[3] / 8)


def test_bands_keep_the_fast_pairs_and_slow_the_slow_ones():
    f, _ = pk.rotary_frequencies(128, 500000.0)
    g, factor = pk.rotary_frequencies(128, 500000.0, {"kind": "bands", "factor": 8.0, "low": 1.0, "high": 4.0, "context": 8192})
    turns = 8192 * np.array(f) / (2 * np.pi)
    ratio = np.array(g) / np.array(f)
    assert factor == 1.0
    assert np.allclose(ratio[turns >= 4], 1.0) and np.allclose(ratio[turns <= 1], 1 / 8)
    mid = (turns > 1) & (turns < 4)
    keep = (turns[mid] - 1) / 3
    assert mid.any() and np.allclose(ratio[mid], keep + (1 - keep) / 8)


def test_ramp_blends_by_index():
    f, _ = pk.rotary_frequencies(128, 10000.0)
    g, factor = pk.rotary_frequencies(128, 10000.0, {"kind": "ramp", "factor": 4.0, "fast": 32, "slow": 1, "context": 4096})
    ratio = np.array(g) / np.array(f)
    at = lambda n: 128 * math.log(4096 / (2 * math.pi * n)) / (2 * math.log(10000.0))
    first, last = math.floor(at(32)), math.ceil(at(1))
    i = np.arange(64)
    keep = 1 - np.clip((i - first) / (last - first), 0, 1)
    assert np.allclose(ratio, keep + (1 - keep) / 4) and np.isclose(factor, 0.1 * math.log(4.0) + 1)
    assert pk.rotary_frequencies(128, 10000.0, {"kind": "ramp", "factor": 4.0, "fast": 32, "slow": 1, "context": 4096, "attention": 1.5})[1] == 1.5


def test_turns_are_the_frequencies_in_fixed_point():
    r = pk.rotary(64, 500000.0, layout="interleaved", device="cpu")
    f, _ = pk.rotary_frequencies(64, 500000.0)
    turns = [int(t) % 2 ** 64 for t in r.turns]
    assert r.interleaved and r.width == 64
    assert np.allclose(np.array(turns, np.float64) / 2.0 ** 64, np.array(f) / (2 * np.pi), rtol=1e-15)


@pytest.mark.parametrize("kw", [dict(width=8), dict(width=24), dict(width=0), dict(layout="pairs"), dict(base=0.0), dict(base=math.inf),
                                dict(scaling={"factor": 2}), dict(scaling={"kind": "other"}), dict(scaling={"kind": "linear", "factor": 0.5}),
                                dict(scaling={"kind": "linear", "factor": math.nan}), dict(scaling={"kind": "bands", "factor": 2}),
                                dict(scaling={"kind": "linear", "factor": 2, "low": 1}),
                                dict(scaling={"kind": "bands", "factor": 2, "low": 4, "high": 1, "context": 10}),
                                dict(scaling={"kind": "bands", "factor": 2, "low": 1, "high": 4, "context": -1}),
                                dict(scaling={"kind": "ramp", "factor": 2, "fast": 1, "slow": 32, "context": 10})])
def test_rotary_refusals(kw):
    with pytest.raises(ValueError):
        pk.rotary(**{"width": 64, "device": "cpu", **kw})


# ------------------------------------------------------------------ refusals

def _struct(**kw):
    base = dict(S=2, H=3, P=7, M=4, d=128, data=16, bias=0, table=4, len=4, free=4, n_free=4, state=256)
    base.update(kw)
    return binding._Pages4(*[base[n] for n, _ in binding._Pages4._fields_])


def l2(s):
    return None if s is None else (ctypes.c_int64 * 2)(*s)


def _extend(lib, c, N=4, counts=4, starts=4, slots=4, positions=4, flags=1):
    return lib.arckv_pages_extend(ctypes.byref(c), counts, N, starts, slots, positions, flags, None)


def _append(lib, c, N=4, K=16, ks=None, V=16, vs=None, slots=4, bias=None, flags=1):
    return lib.arckv_pages_append(ctypes.byref(c), N, K, l2(ks), V, l2(vs), slots, bias, flags, None)


def _read(lib, c, N=4, slots=4, K=16, V=16, flags=1):
    return lib.arckv_pages_read(ctypes.byref(c), N, slots, K, V, flags, None)


def _attend(lib, c, N=4, G=4, most=4, scale=0.0, Q=16, qs=None, starts=4, O=16, os=None, ws=256, nbytes=1 << 40, flags=1):
    return lib.arckv_pages_attend(ctypes.byref(c), N, G, most, scale, Q, l2(qs), starts, O, l2(os), ws, nbytes, flags, None)


CALLS = {"extend": _extend, "truncate": lambda lib, c, flags=1: lib.arckv_pages_truncate(ctypes.byref(c), 4, flags, None),
         "append": _append, "read": _read, "attend": _attend}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("kw,code", [
    (dict(d=64), UNSUPPORTED), (dict(S=0), SHAPE), (dict(S=4097), SHAPE), (dict(H=0), SHAPE), (dict(H=40000), SHAPE),
    (dict(P=0), SHAPE), (dict(P=(1 << 24) + 1), SHAPE), (dict(M=0), SHAPE), (dict(M=(1 << 20) + 1), SHAPE),
    (dict(S=4096, H=32767, M=17), SHAPE), (dict(data=0), BAD), (dict(data=8), BAD), (dict(table=0), BAD), (dict(table=2), BAD),
    (dict(len=0), BAD), (dict(free=0), BAD), (dict(n_free=0), BAD), (dict(n_free=6), BAD), (dict(bias=8), BAD),
    (dict(state=0), BAD), (dict(state=128), BAD)])
def test_bad_pages_are_refused_by_every_call(lib, name, kw, code):
    assert CALLS[name](lib, _struct(**kw)) == code


@pytest.mark.parametrize("name,kw,code", [
    ("extend", dict(N=-1), SHAPE), ("extend", dict(N=1 << 30), SHAPE), ("extend", dict(counts=None), BAD), ("extend", dict(counts=2), BAD),
    ("extend", dict(starts=None), BAD), ("extend", dict(slots=None), BAD), ("extend", dict(positions=6), BAD), ("extend", dict(flags=4), BAD),
    ("truncate", dict(flags=2), BAD),
    ("append", dict(N=0), SHAPE), ("append", dict(N=1 << 30), SHAPE), ("append", dict(K=None), BAD), ("append", dict(K=24), BAD),
    ("append", dict(V=8), BAD), ("append", dict(ks=(12, 128)), BAD), ("append", dict(vs=(1024, 4)), BAD), ("append", dict(slots=None), BAD),
    ("append", dict(slots=2), BAD), ("append", dict(bias=16), BAD), ("append", dict(flags=8), BAD),
    ("read", dict(N=0), SHAPE), ("read", dict(slots=None), BAD), ("read", dict(K=None, V=None), BAD), ("read", dict(K=8), BAD),
    ("read", dict(V=8), BAD), ("read", dict(flags=0x11), BAD),
    ("attend", dict(N=0), SHAPE), ("attend", dict(G=0), SHAPE), ("attend", dict(G=4097), SHAPE), ("attend", dict(most=0), SHAPE),
    ("attend", dict(most=(1 << 24) + 1), SHAPE), ("attend", dict(G=4096, most=1 << 17), SHAPE), ("attend", dict(scale=-1.0), BAD),
    ("attend", dict(scale=math.nan), BAD), ("attend", dict(scale=math.inf), BAD), ("attend", dict(Q=None), BAD), ("attend", dict(Q=8), BAD),
    ("attend", dict(qs=(4, 512)), BAD), ("attend", dict(os=(2048, 4)), BAD), ("attend", dict(O=None), BAD), ("attend", dict(O=8), BAD),
    ("attend", dict(starts=None), BAD), ("attend", dict(starts=2), BAD), ("attend", dict(ws=None), WS), ("attend", dict(ws=128), WS),
    ("attend", dict(nbytes=4095), WS), ("attend", dict(flags=4), BAD)])
def test_bad_arguments_are_refused(lib, name, kw, code):
    assert CALLS[name](lib, _struct(), **kw) == code


def _rotate(lib, N=4, d=128, r=128, f=1.0, turns=8, positions=4, X=16, xs=None, Y=16, ys=None, heads=1, X2=None, xs2=None, Y2=None, ys2=None,
            heads2=0, flags=0):
    return lib.arckv_rotate(N, d, r, f, turns, positions, X, l2(xs), Y, l2(ys), heads, X2, l2(xs2), Y2, l2(ys2), heads2, flags, None)


@pytest.mark.parametrize("kw,code", [
    (dict(d=120), UNSUPPORTED), (dict(d=528), UNSUPPORTED), (dict(r=0), UNSUPPORTED), (dict(r=24), UNSUPPORTED), (dict(d=64), UNSUPPORTED),
    (dict(N=0), SHAPE), (dict(N=1 << 30), SHAPE), (dict(turns=None), BAD), (dict(turns=4), BAD), (dict(positions=None), BAD),
    (dict(positions=2), BAD), (dict(f=math.inf), BAD), (dict(X=None), BAD), (dict(X=24), BAD), (dict(Y=None), BAD),
    (dict(Y=8), BAD), (dict(heads=0), SHAPE), (dict(heads=65536), SHAPE), (dict(xs=(4, 128)), BAD), (dict(ys=(128, 4)), BAD),
    (dict(xs=(128, 128), ys=(256, 128)), BAD), (dict(ys=(256, 128)), BAD), (dict(X2=32), BAD), (dict(Y2=32), BAD),
    (dict(X2=32, Y2=32), SHAPE), (dict(X2=32, Y2=40, heads2=1), BAD), (dict(X2=32, Y2=64, heads2=1, xs2=(2, 128)), BAD), (dict(flags=8), BAD)])
def test_bad_rotations_are_refused(lib, kw, code):
    assert _rotate(lib, **kw) == code


def test_workspace_sizes(lib):
    size = lib.arckv_pages_attend_workspace_bytes
    assert size(2, 3, 4, 128, 1, 4) >= pk.CACHE_WS_HEADER
    assert size(2, 3, 4, 64, 1, 4) == 0 and size(2, 3, 4, 128, 0, 4) == 0 and size(0, 3, 4, 128, 1, 4) == 0
    assert size(64, 8, 128, 128, 512, 4) < 1 << 30
