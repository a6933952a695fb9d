"""Paged caches held in 4 bits, and rotary positions: argument marshalling for the ``arckv_pages_*`` and ``arckv_rotate``
calls of ``libarckv.so``.  Everything here is reached through the package itself."""
from __future__ import annotations

import ctypes
import dataclasses
import math
from typing import Dict, Optional

import paper_2609_36835_gb300 as _pk

PAGE_TOKENS = 64
PAGE_BYTES = 9472
FLAG_INTERLEAVED = 0x10
FLAG_TRANSPOSE = 0x20

_I64x2 = ctypes.c_int64 * 2


class _Pages4(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("S", "H", "P", "M", "d")] +
                [(n, ctypes.c_void_p) for n in ("data", "bias", "table", "len", "free", "n_free", "state")])


def _declare(lib) -> None:
    """Argument types of the library's entries."""
    I, P, U, C, L2 = ctypes.c_int32, ctypes.c_void_p, ctypes.c_uint32, ctypes.POINTER(_Pages4), ctypes.POINTER(_I64x2)
    for name, args in (("arckv_pages_extend", [C, P, I, P, P, P, U, P]), ("arckv_pages_truncate", [C, P, U, P]),
                       ("arckv_pages_append", [C, I, P, L2, P, L2, P, P, U, P]), ("arckv_pages_read", [C, I, P, P, P, U, P]),
                       ("arckv_pages_attend", [C, I, I, I, ctypes.c_float, P, L2, P, P, L2, P, ctypes.c_size_t, U, P]),
                       ("arckv_rotate", [I, I, I, ctypes.c_float, P, P, P, L2, P, L2, I, P, L2, P, L2, I, U, P])):
        entry = getattr(lib, name)
        entry.argtypes, entry.restype = args, ctypes.c_int
    lib.arckv_pages_attend_workspace_bytes.argtypes = [I] * 6
    lib.arckv_pages_attend_workspace_bytes.restype = ctypes.c_size_t


@dataclasses.dataclass(frozen=True, eq=False)
class Pages4:
    """A pool of 4-bit pages and the requests that use it (mirrors ``arckv_pages4``; the header has what the pages hold).
    ``pages_alloc`` makes an empty one; the tensors stay the caller's and are not replaced."""
    data: object                  # uint8 [P, H, 9472]
    table: object                 # int32 [S, M], pages of each request, -1 for none
    len: object                   # int32 [S], tokens of each request
    free: object                  # int32 [P], the free pages first
    n_free: object                # int32 [1]
    bias: object = None           # fp32 [P, H, 64] or None
    state: object = None          # uint8 [256], made here unless given

    def __post_init__(self):
        import torch
        i32 = (torch.int32,)
        _pk._expect("data", self.data, (torch.uint8,), (None, None, PAGE_BYTES))
        P, H, _ = self.data.shape
        _pk._expect("table", self.table, i32, (None, None))
        S, M = self.table.shape
        _pk._expect("len", self.len, i32, (S,))
        _pk._expect("free", self.free, i32, (P,))
        _pk._expect("n_free", self.n_free, i32, (1,))
        if self.bias is not None:
            _pk._expect("bias", self.bias, (torch.float32,), (P, H, PAGE_TOKENS))
        if self.state is None:
            object.__setattr__(self, "state", torch.zeros(256, dtype=torch.uint8, device=self.data.device))
        _pk._expect("state", self.state, (torch.uint8,), (256,))
        _pk._on_one_cuda_device(data=self.data, table=self.table, len=self.len, free=self.free, n_free=self.n_free,
                                bias=self.bias, state=self.state)
        object.__setattr__(self, "_c", _Pages4(S, H, P, M, 128, *[_pk._ptr(getattr(self, n)) for n, _ in _Pages4._fields_[5:]]))
        object.__setattr__(self, "_ref", ctypes.byref(self._c))
        object.__setattr__(self, "_alone", torch.cuda.device_count() == 1)   # no other device can be the current one

    def _tensors(self):
        """All arrays that the calls read or write."""
        return [getattr(self, n) for n, _ in _Pages4._fields_[5:]]

    def _entry(self, name):
        """The library's entry `name`, to be called with the pages' device current."""
        call = getattr(_pk.load_library(), name)
        return call if self._alone else _pk._on_device(self.data.device, call)


def pages_alloc(S: int, H: int, n_pages: int, max_len: int, *, bias: bool = False, device="cuda") -> Pages4:
    """A pool of n_pages pages of 64 tokens and H KV heads for S requests of up to max_len tokens, none of which has any
    yet; with `bias` it holds a logit bias for each token (the beta of a compact cache)."""
    import torch
    M = max(1, -(-max_len // PAGE_TOKENS))
    def i32(*shape, value):
        return torch.full(shape, value, dtype=torch.int32, device=device)
    return Pages4(data=torch.empty(n_pages, H, PAGE_BYTES, dtype=torch.uint8, device=device), table=i32(S, M, value=-1),
                  len=i32(S, value=0), free=torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device),
                  n_free=i32(1, value=n_pages),
                  bias=torch.empty(n_pages, H, PAGE_TOKENS, dtype=torch.float32, device=device) if bias else None)


def pages_workspace(pages: Pages4, max_count: int, G: int):
    """A workspace for ``pages_attend`` with up to max_count rows of a request and G query heads a KV head.  Calls that may
    run at the same time need one each."""
    import torch
    c = pages._c
    need = int(_pk.load_library().arckv_pages_attend_workspace_bytes(c.S, c.H, c.M, c.d, _int32("max_count", max_count), _int32("G", G)))
    if need == 0:
        raise _pk.ArckvError(2, "arckv_pages_attend_workspace_bytes")
    ws = torch.empty(need, dtype=torch.uint8, device=pages.data.device)
    ws[:_pk.CACHE_WS_HEADER].zero_()
    return ws


def _int32(name: str, x: int) -> int:
    if not (_pk._LEAST <= x <= _pk._MOST):
        raise ValueError("arckv: %s out of range: %s" % (name, x))
    return x


def _index(name: str, x, shape, device):
    """Address of a dense int32 tensor of one dimension, of `shape` (None: any), on `device`."""
    import torch
    if (isinstance(x, torch.Tensor) and x.dtype == torch.int32 and (x.shape == shape if shape is not None else x.dim() == 1)
            and x.device == device and x.is_contiguous()):
        return x.data_ptr()
    got = "%s %s on %s" % (x.dtype, tuple(x.shape), x.device) if isinstance(x, torch.Tensor) else type(x).__name__
    raise ValueError("arckv: %s must be a dense int32 tensor of shape %s on %s, got %s" % (name, shape or ("*",), device, got))


def _strides2(name: str, x, dense_from: int):
    """The first two strides of x (None when it is dense), whose dimensions from `dense_from` on must be dense."""
    if x.is_contiguous():
        return None
    st, want = x.stride(), 1
    for i in range(x.dim() - 1, dense_from - 1, -1):
        if st[i] != want and x.shape[i] != 1:
            raise ValueError("arckv: the last %d dimensions of %s must be dense, got strides %s" % (x.dim() - dense_from, name, st))
        want *= x.shape[i]
    return _I64x2(*[st[i] if x.shape[i] != 1 else 0 for i in range(2)])


def _raise_for(st: int, entry: str) -> None:
    if st != 0:
        raise _pk.ArckvError(st, entry)


def pages_extend(pages: Pages4, counts, n_rows: int, *, stream=None, check: bool = True):
    """Make room for counts[s] (int32 [S]) new tokens of every request.  Returns starts [S + 1], the first row of each
    request among the call's packed n_rows rows, and for each row its slot and its position [n_rows]; rows behind the last
    request have -1.  A request that does not fit (table, pool or rows) is left as it is, with slots of -1; it keeps its rows
    in starts, and what ``pages_attend`` writes there means nothing.  The others are extended all the same: the error that
    this raises then has the three results as its `rows` (to go on with those that fit, or to take them back with
    ``pages_truncate``).
    With check=False the call only enqueues, and ``arckv_query_status(pages.state)`` reports errors."""
    import torch
    c, dev = pages._c, pages.data.device
    counts_ptr = _index("counts", counts, (c.S,), dev)
    if not 0 <= n_rows < 1 << 30:
        raise ValueError("arckv: n_rows out of range: %s" % n_rows)
    if stream is not None:   # the outputs belong to the stream that fills them
        stream = _pk._side_stream(stream, dev, counts, *pages._tensors())
        with torch.cuda.stream(stream):
            return pages_extend(pages, counts, n_rows, check=check)
    i32 = torch.int32   # (half of the call's host time; new_empty takes twice as long, one allocation cut in three too)
    starts = torch.empty((c.S + 1,), dtype=i32, device=dev)
    slots, positions = torch.empty((n_rows,), dtype=i32, device=dev), torch.empty((n_rows,), dtype=i32, device=dev)
    st = pages._entry("arckv_pages_extend")(
        pages._ref, counts_ptr, n_rows, starts.data_ptr(), slots.data_ptr(), positions.data_ptr(),
        0 if check else _pk.FLAG_NONBLOCKING, _pk._current_handle(dev))
    if st != 0:
        error = _pk.ArckvError(st, "arckv_pages_extend")
        error.rows = (starts, slots, positions) if check and st in (1, 2) and _sound(c) else None
        raise error
    return starts, slots, positions


def _sound(c: _Pages4) -> bool:
    """Whether the library takes these pages at all: an error of a call on them was then found by its kernel."""
    sizes = _pk.load_library().arckv_pages_attend_workspace_bytes(c.S, c.H, c.M, c.d, 1, 1) > 0 and 1 <= c.P <= 1 << 24
    return sizes and not any((getattr(c, n) or 0) % to for n, to in (("data", 16), ("bias", 16), ("state", 256)))


def pages_truncate(pages: Pages4, lens, *, stream=None, check: bool = True) -> None:
    """Shorten every request to lens[s] tokens (int32 [S]; zero ends it) and give the pages behind them back."""
    c, dev = pages._c, pages.data.device
    lens_ptr = _index("lens", lens, (c.S,), dev)
    handle = _pk._current_handle(dev) if stream is None else _pk._side_stream(stream, dev, lens, *pages._tensors()).cuda_stream
    _raise_for(pages._entry("arckv_pages_truncate")(pages._ref, lens_ptr, 0 if check else _pk.FLAG_NONBLOCKING, handle),
               "arckv_pages_truncate")


def pages_append(pages: Pages4, K, V, slots, *, bias=None, stream=None, check: bool = True) -> None:
    """Write the rows K, V [N, H, 128] (bf16 or fp32, dense in the last dimension) at their slots (int32 [N], distinct;
    those below zero are passed over).  bias [N, H]: their logit biases (zeros when not given).
    With check=False the call only enqueues, and ``arckv_query_status(pages.state)`` reports errors."""
    import torch
    c, dev, shape, dtype = pages._c, pages.data.device, K.shape, K.dtype
    if (len(shape) != 3 or shape[1] != c.H or shape[2] != 128 or V.shape != shape or V.dtype != dtype
            or (dtype != torch.bfloat16 and dtype != torch.float32)):
        raise ValueError("arckv: K and V must be bfloat16 or float32 of shape %s, got %s %s and %s %s"
                         % (("n", c.H, 128), dtype, tuple(shape), V.dtype, tuple(V.shape)))
    if K.device != dev or V.device != dev:
        raise ValueError("arckv: K is on %s, V on %s but the pages on %s" % (K.device, V.device, dev))
    N = shape[0]
    slots_ptr = _index("slots", slots, (N,), dev)
    if bias is not None:
        if pages.bias is None:
            raise ValueError("arckv: these pages hold no bias")
        _pk._expect("bias", bias, (torch.float32,), (N, c.H))
        if bias.device != dev:
            raise ValueError("arckv: bias is on %s but the pages on %s" % (bias.device, dev))
    ks, vs = _strides2("K", K, 2), _strides2("V", V, 2)
    if N == 0:
        return
    handle = (_pk._current_handle(dev) if stream is None else
              _pk._side_stream(stream, dev, K, V, slots, bias, *pages._tensors()).cuda_stream)
    flags = (0 if check else _pk.FLAG_NONBLOCKING) | (_pk.FLAG_F32 if dtype == torch.float32 else 0)
    _raise_for(pages._entry("arckv_pages_append")(pages._ref, N, K.data_ptr(), ks, V.data_ptr(), vs, slots_ptr, _pk._ptr(bias),
                                                  flags, handle), "arckv_pages_append")


def pages_read(pages: Pages4, slots, *, dtype=None, stream=None, check: bool = True):
    """The values that the rows at `slots` (int32 [N]) stand for, as a pair K, V [N, H, 128] in bf16 (or
    dtype=torch.float32); rows of slots below zero are zero."""
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("arckv: dtype must be torch.bfloat16 or torch.float32, got %s" % dtype)
    c, dev = pages._c, pages.data.device
    slots_ptr = _index("slots", slots, None, dev)
    if stream is not None:
        stream = _pk._side_stream(stream, dev, slots, *pages._tensors())
        with torch.cuda.stream(stream):
            return pages_read(pages, slots, dtype=dtype, check=check)
    N = slots.shape[0]
    K = torch.empty((N, c.H, 128), dtype=dtype, device=dev)
    V = torch.empty_like(K)
    if N > 0:
        flags = (0 if check else _pk.FLAG_NONBLOCKING) | (_pk.FLAG_F32 if dtype == torch.float32 else 0)
        _raise_for(pages._entry("arckv_pages_read")(pages._ref, N, slots_ptr, K.data_ptr(), V.data_ptr(), flags,
                                                    _pk._current_handle(dev)), "arckv_pages_read")
    return K, V


def pages_attend(pages: Pages4, Q, starts, logit_scale: float = 0.0, *, max_count: Optional[int] = None, causal: bool = True,
                 out=None, ws=None, stream=None, check: bool = True):
    """O = softmax(scale Q K^T + bias) V for packed queries Q [N, H, G, 128] bf16 (the last two dimensions dense): rows
    starts[s] .. starts[s + 1] - 1 read the pages of request s.  causal: they are its newest tokens, and each sees the
    tokens up to itself.  Returns bf16 of Q's shape, or fills `out`; rows of no request are left as they are (in a tensor
    made here: undefined).  max_count: the most rows of a request (N unless given); few rows take a lighter path.
    ws: a ``pages_workspace`` for max_count, kept by programs that call often.  With check=False the call only enqueues,
    and ``arckv_query_status(ws)`` reports errors: of a workspace made here they are lost."""
    import torch
    c, dev, shape = pages._c, pages.data.device, Q.shape
    if len(shape) != 4 or Q.dtype != torch.bfloat16 or shape[1] != c.H or shape[3] != 128:
        raise ValueError("arckv: Q must be bfloat16 of shape %s, got %s %s" % (("n", c.H, "G", 128), Q.dtype, tuple(shape)))
    if Q.device != dev:
        raise ValueError("arckv: Q is on %s but the pages on %s" % (Q.device, dev))
    starts_ptr = _index("starts", starts, (c.S + 1,), dev)
    N, G = shape[0], shape[2]
    if max_count is None:
        max_count = max(N, 1)
    _int32("max_count", max_count)
    if stream is not None:   # a workspace and an output made here belong to the stream that fills them
        stream = _pk._side_stream(stream, dev, Q, starts, out, ws, *pages._tensors())
        with torch.cuda.stream(stream):
            return pages_attend(pages, Q, starts, logit_scale, max_count=max_count, causal=causal, out=out, ws=ws, check=check)
    if out is None:
        out = torch.empty(shape, dtype=torch.bfloat16, device=dev)
    elif not isinstance(out, torch.Tensor) or out.dtype != torch.bfloat16 or out.shape != shape or out.device != dev:
        raise ValueError("arckv: out must be bfloat16 of shape %s on %s" % (tuple(shape), dev))
    elif not out.is_contiguous() and not _pk._apart(out):
        raise ValueError("arckv: rows of out share memory, strides %s" % (tuple(out.stride()),))
    if ws is None:
        ws = pages_workspace(pages, max_count, G)
    elif not isinstance(ws, torch.Tensor) or ws.dtype != torch.uint8 or ws.device != dev or not ws.is_contiguous():
        raise ValueError("arckv: ws must be a dense uint8 tensor on %s (pages_workspace makes one)" % dev)
    qs, os = _strides2("Q", Q, 2), _strides2("out", out, 2)
    if N == 0:
        return out
    flags = (0 if check else _pk.FLAG_NONBLOCKING) | (_pk.FLAG_CAUSAL if causal else 0)
    _raise_for(pages._entry("arckv_pages_attend")(
        pages._ref, N, G, max_count, logit_scale, Q.data_ptr(), qs, starts_ptr, out.data_ptr(), os, ws.data_ptr(), ws.numel(),
        flags, _pk._current_handle(dev)), "arckv_pages_attend")
    return out


# ------------------------------------------------------------- rotary positions

@dataclasses.dataclass(frozen=True, eq=False)
class Rotary:
    """How ``rotate`` turns the first `width` elements of a head; ``rotary`` makes one."""
    turns: object                 # int64 [width / 2]: turns a position in units of 2^-64, as unsigned bits
    factor: float = 1.0           # of the turned elements
    interleaved: bool = False     # pairs (2i, 2i + 1) instead of (i, i + width / 2)

    def __post_init__(self):
        import torch
        _pk._expect("turns", self.turns, (torch.int64,), (None,))
        if self.turns.shape[0] < 8 or self.turns.shape[0] % 8:
            raise ValueError("arckv: the width must be a positive multiple of 16, got %d" % (2 * self.turns.shape[0]))
        if not math.isfinite(self.factor):
            raise ValueError("arckv: the factor must be finite, got %s" % self.factor)

    @property
    def width(self) -> int:
        return 2 * self.turns.shape[0]


def rotary_frequencies(width: int, base: float = 10000.0, scaling: Optional[Dict[str, object]] = None):
    """Radians a position of each of width / 2 pairs, base^(-2i / width) scaled for long contexts, and the factor of the
    turned elements, as (list of floats, float).  scaling: None, or a dict with "kind" and
      linear  factor: all by 1 / factor
      base    factor: the base grows by factor^(width / (width - 2)), so that the slowest pair slows down by the factor
              and the fastest keeps its speed
      bands   factor, low, high, context: pairs with fewer than `low` turns over `context` positions by 1 / factor, with
              more than `high` as they are, blended by turns in between
      ramp    factor, fast, slow, context (attention): as bands, but blended by the pair's index between those of `fast`
              and `slow` turns; attention: the factor of the turned elements, 0.1 ln(factor) + 1 unless given"""
    if width < 2 or width % 2:
        raise ValueError("arckv: the width must be even, got %s" % width)
    if not (base > 0 and math.isfinite(base)):
        raise ValueError("arckv: the base must be positive, got %s" % base)
    rest = dict(scaling or {})
    kind, factor = rest.pop("kind", None), float(rest.pop("factor", 1.0))
    keys = {None: (), "linear": (), "base": (), "bands": ("low", "high", "context"), "ramp": ("fast", "slow", "context")}
    if kind not in keys or (scaling is not None and kind is None):
        raise ValueError("arckv: unknown scaling %r" % (scaling,))
    if not (factor >= 1.0 and math.isfinite(factor)):
        raise ValueError("arckv: the scaling's factor must be at least 1, got %s" % factor)
    attention = rest.pop("attention", None) if kind == "ramp" else None
    if set(rest) != set(keys[kind]):
        raise ValueError("arckv: scaling %r takes %s" % (kind, ("factor",) + keys[kind]))
    if any(not (isinstance(v, (int, float)) and v > 0 and math.isfinite(v)) for v in rest.values()):
        raise ValueError("arckv: the scaling's parameters must be positive, got %r" % (scaling,))
    if kind == "base" and width > 2:
        base = base * factor ** (width / (width - 2))
    f = [base ** (-2.0 * i / width) for i in range(width // 2)]
    if kind == "linear":
        return [x / factor for x in f], 1.0
    if kind == "bands":
        low, high = float(rest["low"]), float(rest["high"])
        if not low < high:
            raise ValueError("arckv: low must be below high, got %s and %s" % (low, high))
        keep = [min(max((rest["context"] * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
    elif kind == "ramp":
        if not rest["slow"] < rest["fast"] or base <= 1.0:
            raise ValueError("arckv: slow must be below fast and the base above 1, got %r, base %s" % (scaling, base))
        # (real) index of the pair that makes n turns over the context
        def at(n):
            return width * math.log(rest["context"] / (2 * math.pi * n)) / (2 * math.log(base))
        first = max(math.floor(at(rest["fast"])), 0)
        last = max(min(math.ceil(at(rest["slow"])), width - 1), first)
        keep = [1.0 - min(max((i - first) / max(last - first, 0.001), 0.0), 1.0) for i in range(width // 2)]
    else:
        return f, 1.0
    scale = 1.0
    if kind == "ramp":
        scale = 0.1 * math.log(factor) + 1.0 if attention is None else float(attention)
    return [x * k + x / factor * (1.0 - k) for x, k in zip(f, keep)], scale


def rotary(width: int, base: float = 10000.0, *, layout: str = "half", scaling: Optional[Dict[str, object]] = None,
           device="cuda") -> Rotary:
    """Rotary positions over the first `width` elements of a head (a multiple of 16), pairs (i, i + width / 2) for the
    layout "half" and (2i, 2i + 1) for "interleaved"; base and scaling as for ``rotary_frequencies``."""
    import torch
    if layout not in ("half", "interleaved"):
        raise ValueError('arckv: layout must be "half" or "interleaved", got %r' % (layout,))
    if width < 16 or width % 16:
        raise ValueError("arckv: the width must be a positive multiple of 16, got %s" % width)
    freq, factor = rotary_frequencies(width, base, scaling)
    # turns a position mod 1 in units of 2^-64; the division by 2 pi is exact to 2^-53 of the frequency
    bits = [int(round(math.ldexp(math.modf(f / (2 * math.pi))[0], 64))) & (2 ** 64 - 1) for f in freq]
    signed = [b - 2 ** 64 if b >= 2 ** 63 else b for b in bits]
    return Rotary(torch.tensor(signed, dtype=torch.int64, device=device), factor, layout == "interleaved")


def rotate(how: Rotary, positions, X, X2=None, *, out=None, transpose: bool = False, stream=None):
    """X, and X2 if given, with each row's head turned by its position (int32 [N]; rows with one below zero are copied):
    [N, heads, d] bf16 or fp32, dense in the last dimension, d a multiple of 16 up to 512, both of one type and d.
    Returns new tensors (a pair when X2 is given), or fills `out` (a tensor or a pair), which may be X and X2 themselves.
    transpose: the transposed map, which takes gradients of the outputs to those of X and X2 (autograd does not record the
    call, as none of this package)."""
    import torch
    dev, dtype = X.device, X.dtype
    if X.dim() != 3 or (dtype != torch.bfloat16 and dtype != torch.float32):
        raise ValueError("arckv: X must be bfloat16 or float32 of shape ('n', 'heads', 'd'), got %s %s" % (dtype, tuple(X.shape)))
    N, heads, d = X.shape
    heads2 = 0
    if X2 is not None:
        if X2.dim() != 3 or X2.dtype != dtype or X2.shape[0] != N or X2.shape[2] != d or X2.device != dev:
            raise ValueError("arckv: X2 must be %s of shape %s on %s, got %s %s on %s"
                             % (dtype, (N, "heads", d), dev, X2.dtype, tuple(X2.shape), X2.device))
        heads2 = X2.shape[1]
    if dev.type != "cuda":
        raise ValueError("arckv: X must be on a CUDA device, got %s (there is no CPU path)" % dev)
    turns = how.turns
    width = 2 * turns.shape[0]
    if d % 16 or d > 512 or width > d:
        raise ValueError("arckv: d must be a multiple of 16 up to 512 and at least the width %d, got %d" % (width, d))
    if turns.device != dev:
        raise ValueError("arckv: the rotary's turns are on %s but X on %s" % (turns.device, dev))
    positions_ptr = _index("positions", positions, (N,), dev)
    if stream is not None:   # outputs made here belong to the stream that fills them
        given = out if isinstance(out, (tuple, list)) else (out,)
        stream = _pk._side_stream(stream, dev, turns, positions, X, X2, *given)
        with torch.cuda.stream(stream):
            return rotate(how, positions, X, X2, out=out, transpose=transpose)
    if out is None:
        Y = torch.empty((N, heads, d), dtype=dtype, device=dev)
        Y2 = None if X2 is None else torch.empty((N, heads2, d), dtype=dtype, device=dev)
        ys = ys2 = None
    else:
        if X2 is None:
            Y, Y2 = out[0] if isinstance(out, (tuple, list)) and len(out) == 1 else out, None
        elif isinstance(out, (tuple, list)) and len(out) == 2:
            Y, Y2 = out
        else:
            raise ValueError("arckv: out must be a pair of tensors")
        ys, ys2 = _rotated("out", X, Y), None if X2 is None else _rotated("out's second", X2, Y2)
    result = Y if X2 is None else (Y, Y2)
    xs, xs2 = _strides2("X", X, 2), None if X2 is None else _strides2("X2", X2, 2)
    if heads2 == 0:
        X2 = None
    if heads == 0:   # the second tensor alone
        X, xs, Y, ys, heads, X2 = X2, xs2, Y2, ys2, heads2, None
    if N == 0 or X is None:
        return result
    flags = ((_pk.FLAG_F32 if dtype == torch.float32 else 0) | (FLAG_INTERLEAVED if how.interleaved else 0)
             | (FLAG_TRANSPOSE if transpose else 0))
    second = (None, None, None, None, 0) if X2 is None else (X2.data_ptr(), xs2, Y2.data_ptr(), ys2, heads2)
    entry = _pk._on_device(dev, _pk.load_library().arckv_rotate)
    _raise_for(entry(N, d, width, how.factor, turns.data_ptr(), positions_ptr, X.data_ptr(), xs, Y.data_ptr(), ys, heads, *second,
                     flags, _pk._current_handle(dev)), "arckv_rotate")
    return result


def _rotated(name: str, x, y):
    """Strides of an output y of ``rotate`` for x, which it must match."""
    import torch
    if not isinstance(y, torch.Tensor) or y.dtype != x.dtype or y.shape != x.shape or y.device != x.device:
        raise ValueError("arckv: %s must be %s of shape %s on %s" % (name, x.dtype, tuple(x.shape), x.device))
    if not y.is_contiguous() and not _pk._apart(y):
        raise ValueError("arckv: rows of %s share memory, strides %s" % (name, tuple(y.stride())))
    if y.data_ptr() == x.data_ptr() and y.stride() != x.stride() and y.numel() > 0:
        raise ValueError("arckv: %s in place must have its input's strides, got %s and %s" % (name, y.stride(), x.stride()))
    return _strides2(name, y, 2)
