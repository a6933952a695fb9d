"""GB300-native ARC-KV per-context KV-cache compaction.

A thin ctypes binding over ``libarckv.so`` (C ABI in ``include/arckv.h``).
The functions here only marshal arguments: every step of the compaction
runs in the library's CUDA kernels for sm_103a.  PyTorch tensors are used for
device memory and streams.  There is no CPU fallback: if the library is not
built, every call raises.
"""
from __future__ import annotations

import ctypes
import dataclasses
from pathlib import Path
from typing import Dict, Optional, Sequence

__all__ = [
    "Config", "ArckvError", "STATUS", "NUM_STAGES", "STAGE_NAMES", "load_library", "workspace_bytes", "anchor_count",
    "attend_workspace_bytes", "arckv_compact", "arckv_attend", "arckv_query_status", "status_string",
    "compact_layer", "attend", "INDEXER_FIELDS", "attend_joint", "arckv_attend_joint",
    "attend_joint_workspace_bytes", "FLAG_COMPACT_BF16", "truncated_error", "arckv_truncated_error", "SELECTOR_INDEXER", "SELECTOR_HA", "SELECTOR_VI",
    "arckv_wait_probe", "Cache8", "cache_alloc", "cache_workspace", "cache_append", "cache_read", "cache_attend",
    "cache_select", "CACHE_BLOCK", "FLAG_F32", "FLAG_CAUSAL", "Pages4", "pages_alloc", "pages_workspace", "pages_extend",
    "pages_truncate", "pages_append", "pages_read", "pages_attend", "PAGE_TOKENS", "PAGE_BYTES", "Rotary", "rotary",
    "rotary_frequencies", "rotate",
]

_LIB_PATH = Path(__file__).resolve().parent / "libarckv.so"
_lib = None

STATUS = {
    0: "ARCKV_OK", 1: "ARCKV_ERR_INVALID_ARG", 2: "ARCKV_ERR_SHAPE", 3: "ARCKV_ERR_WORKSPACE",
    4: "ARCKV_ERR_NOT_SPD", 5: "ARCKV_ERR_NONFINITE", 6: "ARCKV_ERR_TIMEOUT", 7: "ARCKV_ERR_CUDA",
    8: "ARCKV_ERR_UNSUPPORTED",
}
FLAG_NONBLOCKING = 0x1
FLAG_COMPACT_BF16 = 0x2
FLAG_F32 = 0x4
FLAG_CAUSAL = 0x8
CACHE_BLOCK = 64
CACHE_WS_HEADER = 4096
SELECTOR_INDEXER, SELECTOR_HA, SELECTOR_VI = 0, 1, 2
NUM_STAGES = 11
STAGE_NAMES = ("indexer_features", "index_logits", "pool_top_t", "reference_attention", "column_profiles",
               "assignment", "merge", "beta_products", "beta_solve", "value_products", "value_solve")
INDEXER_FIELDS = ("L_q", "L_k", "L_x", "b_x", "U_q", "U_k", "U_v", "L_c", "L_v")


class ArckvError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (%s)" % (where, STATUS.get(code, code), status_string(code)))


class _Config(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in
                 ("H_kv", "G", "T", "d", "n_pos", "d_x", "H_I", "d_I", "d_A", "t", "chunk_len")] +
                [(n, ctypes.c_float) for n in
                 ("lambda_m", "logit_scale", "ridge_w", "ridge_v", "eps_w", "b_min", "b_max")] +
                [("flags", ctypes.c_uint32), ("selector", ctypes.c_int32)])


class _Indexer(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in INDEXER_FIELDS]


class _Aux(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("scores", "anchors", "assign", "anchors_in", "assign_in", "stage_events", "launches")]


class _Cache8(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("S", "H", "cap", "d")] +
                [(n, ctypes.c_void_p) for n in ("K", "V", "k_scale", "v_scale", "bounds", "bias", "tail", "tail_amax",
                                                "len", "state")])


@dataclasses.dataclass
class Config:
    """One layer's compaction problem (mirrors ``arckv_config``)."""
    H_kv: int
    T: int
    n_pos: int
    t: int
    G: int = 4
    d: int = 128
    d_x: int = 4096
    H_I: int = 8
    d_I: int = 128
    d_A: int = 128
    chunk_len: int = 0
    lambda_m: float = 0.25
    logit_scale: float = 0.0
    ridge_w: float = 1e-4
    ridge_v: float = 1e-3
    eps_w: float = 2.0611536e-09  # e^-20
    b_min: float = -20.0
    b_max: float = 20.0
    flags: int = 0
    selector: int = 0             # SELECTOR_INDEXER / SELECTOR_HA / SELECTOR_VI (App. B.1)

    @property
    def n(self) -> int:
        return self.n_pos * self.G

    def c_struct(self) -> _Config:
        return _Config(self.H_kv, self.G, self.T, self.d, self.n_pos, self.d_x, self.H_I, self.d_I, self.d_A,
                       self.t, self.chunk_len, self.lambda_m, self.logit_scale, self.ridge_w, self.ridge_v,
                       self.eps_w, self.b_min, self.b_max, self.flags, self.selector)


def load_library():
    """Load libarckv.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not _LIB_PATH.exists():
        raise RuntimeError("%s is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`"
                           % _LIB_PATH)
    lib = ctypes.CDLL(str(_LIB_PATH))
    P = ctypes.c_void_p
    lib.arckv_workspace_bytes.argtypes = [ctypes.POINTER(_Config)]
    lib.arckv_workspace_bytes.restype = ctypes.c_size_t
    lib.arckv_anchor_count.argtypes = [ctypes.POINTER(_Config)]
    lib.arckv_anchor_count.restype = ctypes.c_int32
    lib.arckv_compact.argtypes = [ctypes.POINTER(_Config), P, P, P, P, ctypes.POINTER(_Indexer), P, P, P,
                                  ctypes.POINTER(_Aux), P, ctypes.c_size_t, P]
    lib.arckv_compact.restype = ctypes.c_int
    lib.arckv_attend_workspace_bytes.argtypes = [ctypes.c_int32] * 4
    lib.arckv_attend_workspace_bytes.restype = ctypes.c_size_t
    lib.arckv_attend.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
                                 P, P, P, P, P, P, ctypes.c_size_t, ctypes.c_uint32, P]
    lib.arckv_attend.restype = ctypes.c_int
    lib.arckv_attend_joint_workspace_bytes.argtypes = [ctypes.c_int32] * 5
    lib.arckv_attend_joint_workspace_bytes.restype = ctypes.c_size_t
    lib.arckv_attend_joint.argtypes = [ctypes.c_int32] * 5 + [ctypes.c_float] + [P] * 8 + [ctypes.c_size_t,
                                                                                         ctypes.c_uint32, P]
    lib.arckv_attend_joint.restype = ctypes.c_int
    lib.arckv_truncated_error_workspace_bytes.argtypes = [ctypes.c_int32] * 5
    lib.arckv_truncated_error_workspace_bytes.restype = ctypes.c_size_t
    lib.arckv_truncated_error.argtypes = [ctypes.c_int32] * 5 + [ctypes.c_float] + [P] * 5 + [P, ctypes.c_size_t,
                                                                                              ctypes.c_uint32, P]
    lib.arckv_truncated_error.restype = ctypes.c_int
    I, L3, C = ctypes.c_int32, ctypes.POINTER(ctypes.c_int64 * 3), ctypes.POINTER(_Cache8)
    for size in (lib.arckv_cache_workspace_bytes, lib.arckv_cache_attend_workspace_bytes,
                 lib.arckv_cache_select_workspace_bytes):
        size.argtypes = [I] * 6
        size.restype = ctypes.c_size_t
    lib.arckv_cache_append.argtypes = [C, I, P, L3, P, L3, P, P, P, ctypes.c_uint32, P]
    lib.arckv_cache_append.restype = ctypes.c_int
    lib.arckv_cache_read.argtypes = [C, I, I, P, P, ctypes.c_uint32, P]
    lib.arckv_cache_read.restype = ctypes.c_int
    lib.arckv_cache_attend.argtypes = [C, I, I, ctypes.c_float, P, L3, P, I, P, L3, P, ctypes.c_size_t,
                                       ctypes.c_uint32, P]
    lib.arckv_cache_attend.restype = ctypes.c_int
    lib.arckv_cache_select.argtypes = [C, I, I, I, I, I, P, L3, P, P, ctypes.c_size_t, ctypes.c_uint32, P]
    lib.arckv_cache_select.restype = ctypes.c_int
    _declare_pages(lib)
    lib.arckv_query_status.argtypes = [P, P]
    lib.arckv_query_status.restype = ctypes.c_int
    lib.arckv_wait_probe.argtypes = [P, ctypes.c_size_t, ctypes.c_uint32, P]
    lib.arckv_wait_probe.restype = ctypes.c_int
    lib.arckv_status_string.argtypes = [ctypes.c_int]
    lib.arckv_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load_library().arckv_status_string(int(code)).decode()


def workspace_bytes(cfg: Config) -> int:
    c = cfg.c_struct()
    return int(load_library().arckv_workspace_bytes(ctypes.byref(c)))


def anchor_count(cfg: Config) -> int:
    """Realized anchors per head t' (App. A.3 chunking; = cfg.t without it), 0 if invalid."""
    c = cfg.c_struct()
    return int(load_library().arckv_anchor_count(ctypes.byref(c)))


def attend_workspace_bytes(H_kv: int, n: int, t: int, d: int = 128) -> int:
    return int(load_library().arckv_attend_workspace_bytes(H_kv, n, t, d))


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not x.is_contiguous():
        # the C ABI takes dense row-major arrays; a strided view would be read with the wrong layout
        raise ValueError("arckv: tensor arguments must be contiguous (row-major); got strides %s"
                         % (tuple(x.stride()),))
    return x.data_ptr()


def _expect(name: str, x, dtypes, shape=None):
    """Check a torch tensor argument of the helpers below: dtype, shape (None
    entries match any extent) and dense layout.  Raises ValueError."""
    import torch
    if not isinstance(x, torch.Tensor):
        raise ValueError("arckv: %s must be a torch tensor" % name)
    if x.dtype not in dtypes:
        raise ValueError("arckv: %s must be %s, got %s" % (name, " or ".join(map(str, dtypes)), x.dtype))
    if shape is not None and (x.dim() != len(shape) or
                              any(w is not None and int(g) != int(w) for g, w in zip(x.shape, shape))):
        raise ValueError("arckv: %s must have shape %s, got %s" % (
            name, tuple("*" if w is None else w for w in shape), tuple(x.shape)))
    if not x.is_contiguous():
        raise ValueError("arckv: %s must be contiguous (row-major)" % name)


def _on_one_cuda_device(**tensors):
    """All given tensors (None entries skipped) on one CUDA device: the
    kernels read them there and there is no CPU path.  Raises ValueError."""
    dev = None
    for name, x in tensors.items():
        if x is None:
            continue
        if x.device.type != "cuda":
            raise ValueError("arckv: %s must be on a CUDA device, got %s (there is no CPU path)" % (name, x.device))
        if dev is not None and x.device != dev:
            raise ValueError("arckv: %s is on %s but the other arguments on %s" % (name, x.device, dev))
        dev = x.device


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def arckv_compact(cfg: Config, K, V, Q_ref, X_ref, idx: Dict[str, object], C_k, beta, C_v, ws, ws_bytes: int,
                  stream=None, scores=None, anchors=None, assign=None, anchors_in=None, assign_in=None,
                  stage_events: Optional[Sequence[int]] = None):
    """Direct binding of ``arckv_compact``.  Tensor arguments may be torch
    tensors or raw device addresses.  Returns (status, launches)."""
    lib = load_library()
    c = cfg.c_struct()
    ix = _Indexer(*[_ptr(idx.get(n)) if idx is not None else None for n in INDEXER_FIELDS])
    launches = ctypes.c_int32(0)
    ev_arr = None
    if stage_events is not None:
        ev_arr = (ctypes.c_void_p * len(stage_events))(*stage_events)
    aux = _Aux(_ptr(scores), _ptr(anchors), _ptr(assign), _ptr(anchors_in), _ptr(assign_in),
               ctypes.cast(ev_arr, ctypes.c_void_p) if ev_arr is not None else None,
               ctypes.cast(ctypes.pointer(launches), ctypes.c_void_p))
    st = lib.arckv_compact(ctypes.byref(c), _ptr(K), _ptr(V), _ptr(Q_ref), _ptr(X_ref), ctypes.byref(ix),
                           _ptr(C_k), _ptr(beta), _ptr(C_v), ctypes.byref(aux), _ptr(ws), int(ws_bytes),
                           _stream_handle(stream))
    return int(st), int(launches.value)


def arckv_attend(H_kv: int, n: int, t: int, d: int, logit_scale: float, Q, C_k, beta, C_v, O, ws, ws_bytes: int,
                 flags: int = 0, stream=None) -> int:
    """Direct binding of ``arckv_attend``; returns the status code."""
    lib = load_library()
    return int(lib.arckv_attend(H_kv, n, t, d, float(logit_scale), _ptr(Q), _ptr(C_k), _ptr(beta), _ptr(C_v),
                                _ptr(O), _ptr(ws), int(ws_bytes), int(flags), _stream_handle(stream)))


def attend_joint_workspace_bytes(H: int, n: int, t: int, F: int, d: int = 128) -> int:
    return int(load_library().arckv_attend_joint_workspace_bytes(H, n, t, F, d))


def arckv_attend_joint(H: int, n: int, t: int, F: int, d: int, logit_scale: float, Q, C_k, beta, C_v, K_fixed,
                       V_fixed, O, ws, ws_bytes: int, flags: int = 0, stream=None) -> int:
    """Direct binding of ``arckv_attend_joint``; returns the status code."""
    lib = load_library()
    return int(lib.arckv_attend_joint(H, n, t, F, d, float(logit_scale), _ptr(Q), _ptr(C_k), _ptr(beta), _ptr(C_v),
                                      _ptr(K_fixed), _ptr(V_fixed), _ptr(O), _ptr(ws), int(ws_bytes), int(flags),
                                      _stream_handle(stream)))


def arckv_truncated_error(H: int, n: int, T: int, t: int, d: int, logit_scale: float, Q_eval, K, V, S, E, ws,
                          ws_bytes: int, flags: int = 0, stream=None) -> int:
    """Direct binding of ``arckv_truncated_error``; returns the status code."""
    lib = load_library()
    return int(lib.arckv_truncated_error(H, n, T, t, d, float(logit_scale), _ptr(Q_eval), _ptr(K), _ptr(V), _ptr(S),
                                         _ptr(E), _ptr(ws), int(ws_bytes), int(flags), _stream_handle(stream)))


def arckv_query_status(ws, stream=None) -> int:
    dev = getattr(ws, "device", None)
    if stream is None and dev is not None and dev.type == "cuda":   # the current stream of its device
        return int(_on_device(dev, load_library().arckv_query_status)(_ptr(ws), _current_handle(dev)))
    return int(load_library().arckv_query_status(_ptr(ws), _stream_handle(stream)))


def arckv_wait_probe(ws, ws_bytes: int, limit_us: int, stream=None) -> int:
    """Direct binding of ``arckv_wait_probe`` (a bounded device wait made to
    give up); returns the status code."""
    return int(load_library().arckv_wait_probe(_ptr(ws), int(ws_bytes), int(limit_us), _stream_handle(stream)))


# ----------------------------------------------------------- torch helpers

def _alloc_ws(nbytes: int, device):
    import torch
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def compact_layer(cfg: Config, K, V, Q_ref, X_ref, idx: Dict[str, object], *, ws=None, anchors_in=None,
                  assign_in=None, want_scores: bool = False, want_anchors: bool = True,
                  want_assign: bool = False, stream=None, stage_events=None, check: bool = True):
    """Allocate outputs (and a workspace unless given) with torch on K's device
    and call ``arckv_compact``.  Returns a dict of tensors plus 'status' and
    'launches'.  Raises ArckvError on a non-OK status when ``check``."""
    import torch
    bf, i32 = (torch.bfloat16,), (torch.int32,)
    H, T, d, n = cfg.H_kv, cfg.T, cfg.d, cfg.n_pos * cfg.G
    _expect("K", K, bf, (H, T, d))
    _expect("V", V, bf, (H, T, d))
    _expect("Q_ref", Q_ref, bf)
    if Q_ref.shape[0] != H or Q_ref.numel() != H * n * d:
        raise ValueError("arckv: Q_ref must hold [H_kv][n_pos * G][d] = %s, got shape %s"
                         % ((H, n, d), tuple(Q_ref.shape)))
    if cfg.selector == SELECTOR_INDEXER and anchors_in is None:
        _expect("X_ref", X_ref, bf, (cfg.n_pos, cfg.d_x))
        for f in INDEXER_FIELDS:
            _expect("indexer." + f, idx.get(f), bf)
            if idx[f].shape[0] != H:
                raise ValueError("arckv: indexer.%s must lead with H_kv = %d, got shape %s"
                                 % (f, H, tuple(idx[f].shape)))
    if anchors_in is not None:
        _expect("anchors_in", anchors_in, i32, (H, anchor_count(cfg)))
    if assign_in is not None:
        _expect("assign_in", assign_in, i32, (H, T))
    checked_idx = {} if not (cfg.selector == SELECTOR_INDEXER and anchors_in is None) else \
        {"X_ref": X_ref, **{"indexer." + f: idx[f] for f in INDEXER_FIELDS}}
    _on_one_cuda_device(K=K, V=V, Q_ref=Q_ref, anchors_in=anchors_in, assign_in=assign_in, **checked_idx)
    dev = K.device
    f32 = dict(dtype=torch.float32, device=dev)
    need = workspace_bytes(cfg)
    if need == 0:
        raise ArckvError(2, "arckv_workspace_bytes")
    if ws is None:
        ws = _alloc_ws(need, dev)
    tp = anchor_count(cfg)
    out = {
        "C_k": torch.empty(cfg.H_kv, tp, cfg.d, **f32),
        "beta": torch.empty(cfg.H_kv, tp, **f32),
        "C_v": torch.empty(cfg.H_kv, tp, cfg.d, **f32),
    }
    if want_scores:
        out["scores"] = torch.empty(cfg.H_kv, cfg.T, **f32)
    if want_anchors:
        out["anchors"] = torch.empty(cfg.H_kv, tp, dtype=torch.int32, device=dev)
    if want_assign:
        out["assign"] = torch.empty(cfg.H_kv, cfg.T, dtype=torch.int32, device=dev)
    st, nl = arckv_compact(cfg, K, V, Q_ref, X_ref, idx, out["C_k"], out["beta"], out["C_v"], ws, ws.numel(),
                           stream=stream, scores=out.get("scores"), anchors=out.get("anchors"),
                           assign=out.get("assign"), anchors_in=anchors_in, assign_in=assign_in,
                           stage_events=stage_events)
    if check and st != 0:
        raise ArckvError(st, "arckv_compact")
    out["status"], out["launches"] = st, nl
    return out


def attend(Q, C_k, beta, C_v, logit_scale: float = 0.0, *, ws=None, stream=None, check: bool = True):
    """O = softmax(scale Q C_k^T + beta) C_v for Q [H, n, 128] bf16 on the device."""
    import torch
    _expect("Q", Q, (torch.bfloat16,), (None, None, None))
    H, n, d = Q.shape
    _expect("C_k", C_k, (torch.float32,), (H, None, d))
    t = C_k.shape[1]
    _expect("beta", beta, (torch.float32,), (H, t))
    _expect("C_v", C_v, (torch.float32,), (H, t, d))
    _on_one_cuda_device(Q=Q, C_k=C_k, beta=beta, C_v=C_v)
    need = attend_workspace_bytes(H, n, t, d)
    if need == 0:
        raise ArckvError(2, "arckv_attend_workspace_bytes")
    if ws is None:
        ws = _alloc_ws(need, Q.device)
    O = torch.empty(H, n, d, dtype=torch.float32, device=Q.device)
    st = arckv_attend(H, n, t, d, logit_scale, Q, C_k, beta, C_v, O, ws, ws.numel(), stream=stream)
    if check and st != 0:
        raise ArckvError(st, "arckv_attend")
    return O


def attend_joint(Q, C_k=None, beta=None, C_v=None, K_fixed=None, V_fixed=None, logit_scale: float = 0.0, *, ws=None,
                 stream=None, check: bool = True):
    """O = softmax(scale Q [C_k; K_fixed]^T + [beta; 0]) [C_v; V_fixed] (App. A.7) for Q [H, n, 128] bf16.
    C_k / C_v fp32 or bf16 (both the same); either block may be omitted."""
    import torch
    _expect("Q", Q, (torch.bfloat16,), (None, None, None))
    H, n, d = Q.shape
    if (C_k is None) != (C_v is None) or (C_k is None) != (beta is None):
        raise ValueError("arckv: C_k, beta and C_v are given together or not at all")
    if (K_fixed is None) != (V_fixed is None):
        raise ValueError("arckv: K_fixed and V_fixed are given together or not at all")
    if C_k is not None:
        _expect("C_k", C_k, (torch.float32, torch.bfloat16), (H, None, d))
        _expect("C_v", C_v, (C_k.dtype,), (H, C_k.shape[1], d))
        _expect("beta", beta, (torch.float32,), (H, C_k.shape[1]))
    if K_fixed is not None:
        _expect("K_fixed", K_fixed, (torch.bfloat16,), (H, None, d))
        _expect("V_fixed", V_fixed, (torch.bfloat16,), (H, K_fixed.shape[1], d))
    _on_one_cuda_device(Q=Q, C_k=C_k, beta=beta, C_v=C_v, K_fixed=K_fixed, V_fixed=V_fixed)
    t = 0 if C_k is None else C_k.shape[1]
    F = 0 if K_fixed is None else K_fixed.shape[1]
    need = attend_joint_workspace_bytes(H, n, t, F, d)
    if need == 0:
        raise ArckvError(2, "arckv_attend_joint_workspace_bytes")
    if ws is None:
        ws = _alloc_ws(need, Q.device)
    flags = FLAG_COMPACT_BF16 if (C_k is not None and C_k.dtype == torch.bfloat16) else 0
    O = torch.empty(H, n, d, dtype=torch.float32, device=Q.device)
    st = arckv_attend_joint(H, n, t, F, d, logit_scale, Q, C_k, beta, C_v, K_fixed, V_fixed, O, ws, ws.numel(),
                            flags=flags, stream=stream)
    if check and st != 0:
        raise ArckvError(st, "arckv_attend_joint")
    return O


def truncated_error(Q_eval, K, V, S, logit_scale: float = 0.0, *, stream=None, check: bool = True):
    """E(S) per head (App. B.1) for Q_eval [H, n, 128], K, V [H, T, 128] bf16 and anchors S [H, t] int32."""
    import torch
    _expect("Q_eval", Q_eval, (torch.bfloat16,), (None, None, None))
    H, n, d = Q_eval.shape
    _expect("K", K, (torch.bfloat16,), (H, None, d))
    T = K.shape[1]
    _expect("V", V, (torch.bfloat16,), (H, T, d))
    if S is not None:
        _expect("S", S, (torch.int32,), (H, None))
    _on_one_cuda_device(Q_eval=Q_eval, K=K, V=V, S=S)
    t = 0 if S is None else S.shape[1]
    need = int(load_library().arckv_truncated_error_workspace_bytes(H, n, T, t, d))
    if need == 0:
        raise ArckvError(2, "arckv_truncated_error_workspace_bytes")
    ws = _alloc_ws(need, Q_eval.device)
    E = torch.empty(H, dtype=torch.float32, device=Q_eval.device)
    st = arckv_truncated_error(H, n, T, t, d, logit_scale, Q_eval, K, V, S, E, ws, ws.numel(), stream=stream)
    if check and st != 0:
        raise ArckvError(st, "arckv_truncated_error")
    return E


# ------------------------------------------------------- caches held in 8 bits

@dataclasses.dataclass(frozen=True, eq=False)
class Cache8:
    """An 8-bit KV cache of S sequences and H KV heads (mirrors ``arckv_cache8``; the header has the layout and what
    the codes stand for).  ``cache_alloc`` makes an empty one; the tensors stay the caller's and are not replaced."""
    K: object                     # uint8 [S, H, cap, 128]
    V: object
    k_scale: object               # fp32 [S, H, cap / 64]
    v_scale: object
    bounds: object                # int8 [S, H, cap / 64, 2, 128]
    tail: object                  # fp32 [S, H, 2, 64, 128]
    tail_amax: object             # fp32 [S, H, 2, 64]
    len: object                   # int32 [S], tokens held
    bias: object = None           # fp32 [S, H, cap] or None
    state: object = None          # uint8 [256], made here unless given

    def __post_init__(self):
        import torch
        u8, f32 = (torch.uint8,), (torch.float32,)
        _expect("K", self.K, u8, (None, None, None, 128))
        S, H, cap, d = self.K.shape
        if cap < CACHE_BLOCK or cap % CACHE_BLOCK:
            raise ValueError("arckv: the capacity must be a positive multiple of %d, got %d" % (CACHE_BLOCK, cap))
        nb = cap // CACHE_BLOCK
        _expect("V", self.V, u8, (S, H, cap, d))
        _expect("k_scale", self.k_scale, f32, (S, H, nb))
        _expect("v_scale", self.v_scale, f32, (S, H, nb))
        _expect("bounds", self.bounds, (torch.int8,), (S, H, nb, 2, d))
        _expect("tail", self.tail, f32, (S, H, 2, CACHE_BLOCK, d))
        _expect("tail_amax", self.tail_amax, f32, (S, H, 2, CACHE_BLOCK))
        _expect("len", self.len, (torch.int32,), (S,))
        if self.bias is not None:
            _expect("bias", self.bias, f32, (S, H, cap))
        if self.state is None:
            object.__setattr__(self, "state", torch.zeros(256, dtype=torch.uint8, device=self.K.device))
        _expect("state", self.state, u8, (256,))
        _on_one_cuda_device(K=self.K, V=self.V, k_scale=self.k_scale, v_scale=self.v_scale, bounds=self.bounds,
                            tail=self.tail, tail_amax=self.tail_amax, len=self.len, bias=self.bias, state=self.state)
        object.__setattr__(self, "_c", _Cache8(S, H, cap, d, *[_ptr(getattr(self, n)) for n, _ in _Cache8._fields_[4:]]))
        object.__setattr__(self, "_ref", ctypes.byref(self._c))
        object.__setattr__(self, "_alone", torch.cuda.device_count() == 1)   # no other device can be the current one

    def _tensors(self):
        """All arrays that the calls read or write."""
        return [getattr(self, n) for n, _ in _Cache8._fields_[4:]]

    def _entry(self, name):
        """The library's entry `name`, to be called with this cache's device current."""
        call = getattr(load_library(), name)
        return call if self._alone else _on_device(self.K.device, call)

    @property
    def capacity(self) -> int:
        return self._c.cap


def cache_alloc(S: int, H: int, capacity: int, *, bias: bool = False, device="cuda") -> Cache8:
    """An empty cache of at least `capacity` tokens for S sequences and H KV heads; with `bias` it holds a logit bias
    for each token (the beta of a compact cache)."""
    import torch
    cap = max(1, -(-capacity // CACHE_BLOCK)) * CACHE_BLOCK
    nb = cap // CACHE_BLOCK
    def e(*shape, dt=torch.float32, f=torch.empty):
        return f(*shape, dtype=dt, device=device)
    return Cache8(K=e(S, H, cap, 128, dt=torch.uint8), V=e(S, H, cap, 128, dt=torch.uint8), k_scale=e(S, H, nb),
                  v_scale=e(S, H, nb), bounds=e(S, H, nb, 2, 128, dt=torch.int8), tail=e(S, H, 2, CACHE_BLOCK, 128),
                  tail_amax=e(S, H, 2, CACHE_BLOCK), len=e(S, dt=torch.int32, f=torch.zeros),
                  bias=e(S, H, cap) if bias else None)


def cache_workspace(cache: Cache8, n_pos: int, G: int):
    """A workspace for ``cache_attend`` and ``cache_select`` with up to n_pos positions of G query heads.  Calls that
    may run at the same time need one each.  (One of either call alone is smaller: the sizes are in the header.)"""
    return _cache_workspace(cache, n_pos, G, "arckv_cache_workspace_bytes")


def _cache_workspace(cache: Cache8, n_pos: int, G: int, size: str):
    import torch
    c = cache._c
    need = int(getattr(load_library(), size)(c.S, c.H, c.cap, c.d, n_pos, G))
    if need == 0:
        raise ArckvError(2, size)
    ws = torch.empty(need, dtype=torch.uint8, device=cache.K.device)
    ws[:CACHE_WS_HEADER].zero_()
    return ws


def _strides3(name: str, x, dense_from: int):
    """The first three strides of x (None when it is dense), whose dimensions from `dense_from` on must be dense."""
    if x.is_contiguous():
        return None
    st = x.stride()
    want = 1
    for i in range(x.dim() - 1, dense_from - 1, -1):
        if st[i] != want and x.shape[i] != 1:
            raise ValueError("arckv: the last %d dimensions of %s must be dense, got strides %s"
                             % (x.dim() - dense_from, name, st))
        want *= x.shape[i]
    return (ctypes.c_int64 * 3)(*[st[i] if x.shape[i] != 1 else 0 for i in range(3)])


_LEAST, _MOST = -0x80000000, 0x7fffffff   # 32-bit integers: of others only the low bits would reach the library


def _apart(x) -> bool:
    """Whether no two elements of x share memory, for a view that slices and permutes a dense tensor."""
    reach = 1
    for st, n in sorted((st, n) for st, n in zip(x.stride(), x.shape) if n > 1):
        if st < reach:
            return False
        reach = st * n
    return True


def _side_stream(stream, device, *tensors):
    """`stream` as a torch stream.  Tensors in use on a stream other than the current one are recorded there, so that
    their memory is not reused too early."""
    import torch
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    if stream != torch.cuda.current_stream(device):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
    return stream


_raw_stream = None


def _current_handle(device) -> int:
    """The raw handle of the device's current stream, without making a stream object where torch has a call for that."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _raw_stream(device.index)


def _on_device(device, call):
    """`call` made with `device` as the current one: the library launches, and sizes its grids, for the current device."""
    import torch
    if torch.cuda.current_device() == device.index:
        return call

    def guarded(*args):
        with torch.cuda.device(device):
            return call(*args)
    return guarded


def _counts_ptr(name: str, x, cache: "Cache8"):
    """Address of an int32 [S] argument on the cache's device, None for none."""
    import torch
    if x is None:
        return None
    if x.dtype != torch.int32 or x.shape != cache.len.shape or x.device != cache.len.device or not x.is_contiguous():
        raise ValueError("arckv: %s must be a dense int32 tensor of shape %s on %s, got %s %s on %s"
                         % (name, tuple(cache.len.shape), cache.len.device, x.dtype, tuple(x.shape), x.device))
    return x.data_ptr()


def cache_append(cache: Cache8, K, V, *, bias=None, at=None, counts=None, stream=None, check: bool = True) -> None:
    """Write the rows K, V [S, H, n, 128] (bf16 or fp32, dense in the last dimension) at the end of every sequence.
    bias [S, H, n]: their logit biases (zeros when not given).  at [S] int32: first token written instead of the end,
    over rejected tokens; it lies in the newest block or is a multiple of 64 (a draft that went on into a new block is
    taken back further by writing the block before again from its first row).  counts [S] int32: how many of the n rows
    each sequence takes.
    With check=False the call only enqueues, and ``arckv_query_status(cache.state)`` reports errors."""
    import torch
    c, dev, shape, dtype = cache._c, cache.K.device, K.shape, K.dtype
    if (len(shape) != 4 or shape[0] != c.S or shape[1] != c.H or shape[3] != 128 or V.shape != shape or V.dtype != dtype
            or (dtype != torch.bfloat16 and dtype != torch.float32)):
        raise ValueError("arckv: K and V must be bfloat16 or float32 of shape %s, got %s %s and %s %s"
                         % ((c.S, c.H, "n", 128), dtype, tuple(shape), V.dtype, tuple(V.shape)))
    if K.device != dev or V.device != dev:
        raise ValueError("arckv: K is on %s, V on %s but the cache on %s" % (K.device, V.device, dev))
    n = shape[2]
    if bias is not None:
        if cache.bias is None:
            raise ValueError("arckv: this cache holds no bias")
        _expect("bias", bias, (torch.float32,), (c.S, c.H, n))
        _on_one_cuda_device(cache=cache.K, bias=bias)
    at_ptr, counts_ptr = _counts_ptr("at", at, cache), _counts_ptr("counts", counts, cache)
    if n == 0:
        return
    handle = (_current_handle(dev) if stream is None else
              _side_stream(stream, dev, K, V, bias, at, counts, *cache._tensors()).cuda_stream)
    flags = (0 if check else FLAG_NONBLOCKING) | (FLAG_F32 if dtype == torch.float32 else 0)
    st = cache._entry("arckv_cache_append")(
        cache._ref, n, K.data_ptr(), _strides3("K", K, 3), V.data_ptr(), _strides3("V", V, 3), _ptr(bias), at_ptr, counts_ptr,
        flags, handle)
    if st != 0:
        raise ArckvError(st, "arckv_cache_append")


def cache_read(cache: Cache8, start: int, count: int, *, dtype=None, stream=None, check: bool = True):
    """The values that `count` tokens from `start` on stand for (negative: from each sequence's end), as a pair
    K, V [S, H, count, 128] in bf16 (or dtype=torch.float32); tokens that a sequence does not hold are zero."""
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("arckv: dtype must be torch.bfloat16 or torch.float32, got %s" % dtype)
    if not (_LEAST <= start <= _MOST and _LEAST <= count <= _MOST):
        raise ValueError("arckv: start, count out of range: %s" % ((start, count),))
    c, dev = cache._c, cache.K.device
    if stream is not None:   # the outputs belong to the stream that fills them
        stream = _side_stream(stream, dev, *cache._tensors())
        with torch.cuda.stream(stream):
            return cache_read(cache, start, count, dtype=dtype, check=check)
    K = torch.empty((c.S, c.H, max(count, 0), 128), dtype=dtype, device=dev)
    V = torch.empty_like(K)
    if count == 0:
        return K, V
    handle = _current_handle(dev)
    flags = (0 if check else FLAG_NONBLOCKING) | (FLAG_F32 if dtype == torch.float32 else 0)
    st = cache._entry("arckv_cache_read")(cache._ref, start, count, K.data_ptr(), V.data_ptr(), flags, handle)
    if st != 0:
        raise ArckvError(st, "arckv_cache_read")
    return K, V


def _check_queries(torch, cache: Cache8, Q):
    """Positions, query heads and device of Q, which must fit the cache."""
    c, shape = cache._c, Q.shape
    if len(shape) != 5 or Q.dtype != torch.bfloat16 or shape[0] != c.S or shape[1] != c.H or shape[4] != 128:
        raise ValueError("arckv: Q must be bfloat16 of shape %s, got %s %s"
                         % ((c.S, c.H, "n_pos", "G", 128), Q.dtype, tuple(shape)))
    dev = cache.K.device
    if Q.device != dev:
        raise ValueError("arckv: Q is on %s but the cache on %s" % (Q.device, dev))
    return shape[2], shape[3], dev


def cache_attend(cache: Cache8, Q, logit_scale: float = 0.0, *, blocks=None, causal: bool = False, out=None, ws=None,
                 stream=None, check: bool = True):
    """O = softmax(scale Q K^T + bias) V over the cache for Q [S, H, n_pos, G, 128] bf16 (the last two dimensions
    dense); returns fp32 of Q's shape and layout, or fills `out`.  causal: the positions are the newest n_pos tokens, and
    each sees the tokens up to itself.  blocks [S, H, n_pos, m] int32: the only blocks that each position reads
    (``cache_select``).  ws: a ``cache_workspace``, kept by programs that call often.  With check=False the call only
    enqueues, and ``arckv_query_status(ws)`` reports errors: of a workspace made here they are lost."""
    import torch
    n_pos, G, dev = _check_queries(torch, cache, Q)
    if stream is not None:   # a workspace and an output made here belong to the stream that fills them
        stream = _side_stream(stream, dev, Q, blocks, out, ws, *cache._tensors())
        with torch.cuda.stream(stream):
            return cache_attend(cache, Q, logit_scale, blocks=blocks, causal=causal, out=out, ws=ws, check=check)
    m, listed = 0, None
    if blocks is not None:
        shape = blocks.shape
        if (len(shape) != 4 or blocks.dtype != torch.int32 or shape[:3] != Q.shape[:3] or shape[3] == 0 or
                blocks.device != dev or not blocks.is_contiguous()):   # (an empty one's address means no list)
            raise ValueError("arckv: blocks must be a dense int32 tensor of shape %s, m >= 1, on %s, got %s %s on %s"
                             % (tuple(Q.shape[:3]) + ("m",), dev, blocks.dtype, tuple(shape), blocks.device))
        m, listed = shape[3], blocks.data_ptr()
    if ws is None:
        ws = _cache_workspace(cache, n_pos, G, "arckv_cache_attend_workspace_bytes")
    elif not isinstance(ws, torch.Tensor) or ws.dtype != torch.uint8 or ws.device != dev or not ws.is_contiguous():
        raise ValueError("arckv: ws must be a dense uint8 tensor on %s (cache_workspace makes one)" % dev)
    if out is None:
        out = torch.empty_like(Q, dtype=torch.float32)
    elif out.dtype != torch.float32 or out.shape != Q.shape or out.device != dev:
        raise ValueError("arckv: out must be float32 of shape %s on %s" % (tuple(Q.shape), dev))
    elif not out.is_contiguous() and not _apart(out):
        raise ValueError("arckv: rows of out share memory, strides %s" % (tuple(out.stride()),))
    handle = _current_handle(dev)
    flags = (0 if check else FLAG_NONBLOCKING) | (FLAG_CAUSAL if causal else 0)
    st = cache._entry("arckv_cache_attend")(
        cache._ref, n_pos, G, logit_scale, Q.data_ptr(), _strides3("Q", Q, 3), listed, m, out.data_ptr(),
        _strides3("out", out, 3), ws.data_ptr(), ws.numel(), flags, handle)
    if st != 0:
        raise ArckvError(st, "arckv_cache_attend")
    return out


def cache_select(cache: Cache8, Q, m: int, *, keep_first: Optional[int] = None, keep_last: int = 1, causal: bool = False,
                 ws=None, stream=None, check: bool = True):
    """The m blocks of 64 tokens that each query position reads, [S, H, n_pos, m] int32 ascending, -1 for none: the
    first keep_first (one where m leaves room for it beside the newest, unless given), the newest keep_last and those
    whose logits can be largest.  Q, causal and ws as for ``cache_attend``."""
    import torch
    n_pos, G, dev = _check_queries(torch, cache, Q)
    if keep_first is None:
        keep_first = 1 if m > keep_last else 0
    if not (_LEAST <= m <= _MOST and _LEAST <= keep_first <= _MOST and _LEAST <= keep_last <= _MOST):
        raise ValueError("arckv: m, keep_first, keep_last out of range: %s" % ((m, keep_first, keep_last),))
    if stream is not None:
        stream = _side_stream(stream, dev, Q, ws, *cache._tensors())
        with torch.cuda.stream(stream):
            return cache_select(cache, Q, m, keep_first=keep_first, keep_last=keep_last, causal=causal, ws=ws,
                                check=check)
    if ws is None:
        ws = _cache_workspace(cache, n_pos, G, "arckv_cache_select_workspace_bytes")
    elif not isinstance(ws, torch.Tensor) or ws.dtype != torch.uint8 or ws.device != dev or not ws.is_contiguous():
        raise ValueError("arckv: ws must be a dense uint8 tensor on %s (cache_workspace makes one)" % dev)
    blocks = torch.empty((cache._c.S, cache._c.H, n_pos, max(m, 0)), dtype=torch.int32, device=dev)
    handle = _current_handle(dev)
    flags = (0 if check else FLAG_NONBLOCKING) | (FLAG_CAUSAL if causal else 0)
    st = cache._entry("arckv_cache_select")(
        cache._ref, n_pos, G, m, keep_first, keep_last, Q.data_ptr(), _strides3("Q", Q, 3), blocks.data_ptr(), ws.data_ptr(),
        ws.numel(), flags, handle)
    if st != 0:
        raise ArckvError(st, "arckv_cache_select")
    return blocks


# paged 4-bit caches and rotary positions (the helpers above are what they share with the calls of this file)
from .pages import (PAGE_BYTES, PAGE_TOKENS, Pages4, Rotary, pages_alloc, pages_append, pages_attend, pages_extend,  # noqa: E402
                    pages_read, pages_truncate, pages_workspace, rotary, rotary_frequencies, rotate)
from .pages import _declare as _declare_pages  # noqa: E402
