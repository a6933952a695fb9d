"""The 8-bit cache without a GPU: its plain form on cases worked out by hand, workspace sizes and refusals on the host."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache8 as ref
import paper_2609_36835_gb300 as pk

BAD, SHAPE, WS, UNSUPPORTED = 1, 2, 3, 8


def test_block_codes_by_hand():
    x = np.zeros((2, 128), np.float32)
    x[0, 0], x[0, 1], x[1, 2] = 127.0, -1.5, 0.5
    codes, scale = ref.quantise_block(x)
    assert scale == np.float32(127.0) * (np.float32(1) / np.float32(127)) and codes[0, 0] == 127
    assert codes[0, 1] == -2 and codes[1, 2] == 0           # halves go to the even code
    zero, s0 = ref.quantise_block(np.zeros((3, 128), np.float32))
    assert not zero.any() and s0 > 0


def test_values_are_within_half_a_step():
    x = np.random.default_rng(0).normal(size=(150, 128)).astype(np.float32)
    codes, scale, bounds = ref.quantise(x)
    step = np.repeat(scale, 64)[:150, None].astype(np.float64)
    assert np.all(np.abs(ref.values(codes, scale) - x) <= 0.5 * step * (1 + 1e-5))
    assert np.array_equal(bounds[2, 0], codes[128:].min(0)) and np.array_equal(bounds[1, 1], codes[64:128].max(0))


def test_scores_bound_the_logits():
    rng = np.random.default_rng(1)
    k, q = rng.normal(size=(640, 128)).astype(np.float32), rng.normal(size=(4, 128)).astype(np.float32)
    codes, scale, bounds = ref.quantise(k)
    qv = np.stack([ref.quantise_block(r[None])[0][0] * np.float64(ref.quantise_block(r[None])[1]) for r in q])
    logits = (qv @ ref.values(codes, scale).T).max(0).reshape(10, 64).max(1)
    assert np.all(ref.block_scores(q, bounds, scale) >= logits - 1e-4)


def test_attention_and_selection_by_hand():
    k, v = np.zeros((130, 4)), np.arange(130.0)[:, None] * np.ones((1, 4))
    q = np.zeros((2, 1, 4))
    assert np.allclose(ref.attend(q, k, v, 1.0)[:, 0, 0], 64.5)
    assert np.allclose(ref.attend(q, k, v, 1.0, causal=True)[:, 0, 0], [64.0, 64.5])
    assert np.allclose(ref.attend(q, k, v, 1.0, blocks=[[2, -1], [-1, -1]])[:, 0, 0], [128.5, 0.0])
    assert not ref.attend(q[:1], k, v, 1.0, bias=np.full(130, -np.inf)).any()
    scale, bounds = np.ones(3, np.float32), np.zeros((3, 2, 4), np.int8)
    bounds[1, 1] = 3
    assert ref.select(np.ones((1, 1, 4)), bounds, scale, 130, 2, 0, 0, False).tolist() == [[0, 1]]
    assert ref.select(np.ones((1, 1, 4)), bounds, scale, 130, 2, 0, 1, False).tolist() == [[1, 2]]
    assert ref.select(np.ones((1, 1, 4)), bounds, scale, 60, 2, 1, 1, False).tolist() == [[0, -1]]


# ------------------------------------------------------------------ refusals

def _struct(**kw):
    base = dict(S=2, H=3, cap=128, d=128, K=16, V=16, k_scale=16, v_scale=16, bounds=16, bias=0, tail=16, tail_amax=16,
                len=16, state=16)
    base.update(kw)
    return pk._Cache8(*[base[n] for n, _ in pk._Cache8._fields_])


def _append(lib, c, n=4, K=16, V=16, ks=None, vs=None, bias=None, flags=1):
    l3 = lambda s: None if s is None else (ctypes.c_int64 * 3)(*s)
    return lib.arckv_cache_append(ctypes.byref(c), n, K, l3(ks), V, l3(vs), bias, None, None, flags, None)


def _attend(lib, c, n_pos=1, G=4, scale=0.0, Q=16, qs=None, blocks=None, m=0, O=16, os=None, ws=256, nbytes=1 << 40,
            flags=1):
    l3 = lambda s: None if s is None else (ctypes.c_int64 * 3)(*s)
    return lib.arckv_cache_attend(ctypes.byref(c), n_pos, G, scale, Q, l3(qs), blocks, m, O, l3(os), ws, nbytes, flags,
                                  None)


def _select(lib, c, m=2, first=1, last=1, blocks=16, n_pos=1, G=4, Q=16, ws=256, nbytes=1 << 40, flags=1):
    return lib.arckv_cache_select(ctypes.byref(c), n_pos, G, m, first, last, Q, None, blocks, ws, nbytes, flags, None)


@pytest.mark.parametrize("kw,code", [
    (dict(d=64), UNSUPPORTED), (dict(S=0), SHAPE), (dict(H=0), SHAPE), (dict(cap=100), SHAPE), (dict(cap=0), SHAPE),
    (dict(S=5000), SHAPE), (dict(cap=1 << 27), SHAPE), (dict(K=0), BAD), (dict(V=8), BAD), (dict(len=0), BAD),
    (dict(state=0), BAD), (dict(bounds=4), BAD), (dict(bias=4), BAD)])
def test_bad_caches_are_refused(lib, kw, code):
    c = _struct(**kw)
    assert _append(lib, c) == code and _attend(lib, c) == code and _select(lib, c) == code
    assert lib.arckv_cache_read(ctypes.byref(c), 0, 1, 16, 16, 1, None) == code


def test_missing_cache_is_refused(lib):
    assert lib.arckv_cache_append(None, 1, 16, None, 16, None, None, None, None, 1, None) == BAD


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), SHAPE), (dict(n=129), SHAPE), (dict(K=None), BAD), (dict(V=None), BAD), (dict(K=8), BAD),
    (dict(ks=(1, 8, 8)), BAD), (dict(vs=(8, 8, 12)), BAD), (dict(bias=16), BAD), (dict(flags=0x9), BAD),
    (dict(flags=0x5, ks=(8, 8, 6)), BAD)])
def test_bad_appends_are_refused(lib, kw, code):
    assert _append(lib, _struct(), **kw) == code


@pytest.mark.parametrize("start,count,K,V,flags,code", [
    (0, 0, 16, 16, 1, SHAPE), (0, -1, 16, 16, 1, SHAPE), (0, 1, None, None, 1, BAD), (0, 1, 8, 16, 1, BAD),
    (0, 1, 16, 16, 0x3, BAD), (1 << 27, 1, 16, 16, 1, SHAPE)])
def test_bad_reads_are_refused(lib, start, count, K, V, flags, code):
    assert lib.arckv_cache_read(ctypes.byref(_struct()), start, count, K, V, flags, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n_pos=0), SHAPE), (dict(G=0), SHAPE), (dict(G=1 << 17), SHAPE), (dict(Q=None), BAD), (dict(Q=8), BAD),
    (dict(qs=(8, 8, 4)), BAD), (dict(O=None), BAD), (dict(os=(4, 2, 4)), BAD), (dict(scale=-1.0), BAD),
    (dict(scale=float("nan")), BAD), (dict(blocks=16, m=0), SHAPE), (dict(ws=None), WS), (dict(ws=128), WS),
    (dict(nbytes=4095), WS), (dict(flags=0x3), BAD)])
def test_bad_attention_is_refused(lib, kw, code):
    assert _attend(lib, _struct(), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(m=0), SHAPE), (dict(m=9000), SHAPE), (dict(first=2), SHAPE), (dict(last=-1), SHAPE), (dict(blocks=None), BAD),
    (dict(blocks=2), BAD), (dict(nbytes=0), WS), (dict(n_pos=-1), SHAPE), (dict(flags=0x5), BAD)])
def test_bad_selections_are_refused(lib, kw, code):
    assert _select(lib, _struct(), **kw) == code


def test_workspace_sizes(lib):
    need = lib.arckv_cache_workspace_bytes(64, 8, 8192, 128, 1, 4)
    assert 64 * 8 * 128 * 4 <= need < 1 << 30
    for bad in ((0, 8, 64, 128, 1, 4), (1, 8, 63, 128, 1, 4), (1, 8, 64, 64, 1, 4), (1, 8, 64, 128, 0, 4),
                (4096, 32767, 1 << 26, 128, 1, 1), (4096, 1024, 64, 128, 1024, 1)):
        assert lib.arckv_cache_workspace_bytes(*bad) == 0


def test_python_calls_refuse_host_tensors_and_wrong_shapes(lib):
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    good = dict(K=z(1, 2, 64, 128, dt=torch.uint8), V=z(1, 2, 64, 128, dt=torch.uint8), k_scale=z(1, 2, 1),
                v_scale=z(1, 2, 1), bounds=z(1, 2, 1, 2, 128, dt=torch.int8), tail=z(1, 2, 2, 64, 128),
                tail_amax=z(1, 2, 2, 64), len=z(1, dt=torch.int32))
    with pytest.raises(ValueError, match="CUDA device"):
        pk.Cache8(**good)
    for name, wrong in (("K", z(1, 2, 60, 128, dt=torch.uint8)), ("V", z(1, 2, 64, 128)), ("k_scale", z(1, 2, 2)),
                        ("bounds", z(1, 2, 1, 128, dt=torch.int8)), ("len", z(2, dt=torch.int32)),
                        ("tail", z(1, 2, 64, 128))):
        with pytest.raises(ValueError):
            pk.Cache8(**{**good, name: wrong})
