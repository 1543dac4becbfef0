"""Operators over a paged key/value cache (C ABI in include/lssvm_cache.h): rotary
positions, writing new tokens, attention, eviction by accumulated weight.

Argument marshalling only, as in the binding of the training path: every step runs
in the HIP library on the current stream of the tensors' device, and nothing is read
back. The calls can be captured into a HIP graph. No gradient is recorded: tensors that
require one are refused unless gradients are off.
"""
from __future__ import annotations

import ctypes
import functools

from ._binding import OK, _check, _workspace, alloc_workspace, lib

F32, BF16, F16 = 1, 2, 3
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


class _Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("pages", ctypes.c_int64), ("heads", ctypes.c_int64), ("page", ctypes.c_int64),
                ("dim", ctypes.c_int64), ("sequences", ctypes.c_int64),
                ("columns", ctypes.c_int64), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("weight_stride", ctypes.c_int64 * 2),
                ("table_stride", ctypes.c_int64), ("dtype", ctypes.c_int32)]


_P, _I64, _I32, _D = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double
_Two = _I64 * 2
_S = ctypes.POINTER(_I64)       # two strides
_C = ctypes.POINTER(_Cache)
_SIGS = {
    "lssvm_rotary_frequencies": (_I32, [_I64, _D, _I32, _D, _D, ctypes.POINTER(_D),
                                        ctypes.POINTER(_D)]),
    "lssvm_rotary": (_I32, [_P, _S, _P, _S, _I64, _I64, _I64, _P, _I32, _P, _I64, _D, _I32,
                            _I32, _I32, _P]),
    "lssvm_cache_append": (_I32, [_C, _P, _S, _P, _S, _I64, _P, _P, _I32, _P, _I64, _D, _I32,
                                  _P]),
    "lssvm_attention_workspace_bytes": (ctypes.c_size_t, [_C, _I64, _I64, _I32]),
    "lssvm_attention": (_I32, [_C, _P, _S, _I64, _I64, _P, _D, _I32, _I32, _P, _S, _P, _S,
                               _P, ctypes.c_size_t, _P]),
    "lssvm_cache_evict": (_I32, [_C, _C, _I64, _I64, _P, _P]),
}


@functools.cache
def _torch():
    import torch
    return torch


@functools.cache
def _lib():
    L = lib()
    for name, (res, args) in _SIGS.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    return L


@functools.cache
def _codes():
    torch = _torch()
    return {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _code(dtype) -> int:
    code = _codes().get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}; use float32, bfloat16 or float16")
    return code


@functools.lru_cache(maxsize=256)
def _two(outer: int, head: int, *_):
    """The first two strides of a tensor, for the library to read."""
    return _Two(outer, head)


def _gpu(t, name: str, dims: int, dtype=None, device=None):
    """t, a GPU tensor of `dims` dimensions with contiguous last one, else an error."""
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dim() != dims:
        raise ValueError(f"{name} must have {dims} dimensions, not {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device}, not {t.device}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t


def _no_gradient(requires_grad: bool) -> None:
    """An error where autograd would be asked to record a call: nothing does that here."""
    if requires_grad and _torch().is_grad_enabled():
        raise ValueError("these calls record no gradient: pass detached tensors or call under "
                         "torch.no_grad() (the gradient of rotary is rotary with transpose)")


@functools.cache
def _raw_stream():
    """The handle of a device's current stream; where torch offers it, without a Stream
    object around it, which costs half as much as a launch."""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _call(device, fn, *args) -> None:
    """The library's call on the device's current stream, with that device current."""
    cuda, index = _torch().cuda, device.index
    if cuda.current_device() == index:
        code = fn(*args, _raw_stream()(index))
    else:
        with cuda.device(device):
            code = fn(*args, _raw_stream()(index))
    if code != OK:
        _check(code)


class PagedCache:
    """Keys and values of sequences in pages of a pool.

    k, v      pages x heads x page x dim, float32, bfloat16 or float16, any strides
              with a contiguous last dimension and rows that begin on 16 bytes
    table     sequences x columns page numbers, int32
    lengths   keys of each sequence, int32
    weight    pages x heads x page, float32: accumulated weight of every key (for
              ``attention(accumulate=True)`` and ``cache_evict``)

    All on one GPU. The cache refers to the tensors: what is written into them is
    seen by the next call. Page numbers outside the pool are holes."""

    def __init__(self, k, v, table, lengths, weight=None):
        torch = _torch()
        _gpu(k, "k", 4)
        code, device = _code(k.dtype), k.device
        _gpu(v, "v", 4, k.dtype, device)
        if v.shape != k.shape:
            raise ValueError(f"v must have the shape of k, {tuple(k.shape)}, not {tuple(v.shape)}")
        _gpu(table, "table", 2, torch.int32, device)
        _gpu(lengths, "lengths", 1, torch.int32, device)
        if lengths.shape[0] != table.shape[0]:
            raise ValueError("lengths needs an entry for each row of table")
        if weight is not None:
            _gpu(weight, "weight", 3, torch.float32, device)
            if weight.shape != k.shape[:3]:
                raise ValueError(f"weight must be {tuple(k.shape[:3])}, not {tuple(weight.shape)}")
        self.k, self.v, self.table, self.lengths, self.weight = k, v, table, lengths, weight
        self.device, self.dtype = device, k.dtype
        self.pages, self.heads, self.page, self.dim = k.shape
        self.sequences, self.columns = table.shape
        self._c = _Cache(
            k.data_ptr(), v.data_ptr(), weight.data_ptr() if weight is not None else None,
            table.data_ptr(), lengths.data_ptr(), *k.shape, *table.shape, k.stride()[:3],
            v.stride()[:3], weight.stride()[:2] if weight is not None else (0, 0),
            table.stride(0), code)
        self._ref = ctypes.byref(self._c)


def _cache(cache, name: str = "cache"):
    if not isinstance(cache, PagedCache):
        raise TypeError(f"{name} must be a PagedCache")
    return cache


def _rows(t, name: str, cache, heads=None):
    _gpu(t, name, 3, cache.dtype, cache.device)
    if t.shape[2] != cache.dim or (heads is not None and t.shape[1] != heads):
        raise ValueError(f"{name} must be tokens x {heads or 'heads'} x {cache.dim}, "
                         f"not {tuple(t.shape)}")
    return t


def _offsets(t, cache):
    _gpu(t, "offsets", 1, _torch().int32, cache.device)
    if t.shape[0] != cache.sequences + 1:
        raise ValueError(f"offsets needs {cache.sequences + 1} entries, not {t.shape[0]}")
    return t.data_ptr()


def _angles(positions, freqs, tokens: int, device):
    """(positions, bytes of one, freqs, pairs) for the library."""
    torch = _torch()
    _no_gradient(_gpu(freqs, "freqs", 1, torch.float64, device).requires_grad)
    _gpu(positions, "positions", 1, None, device)
    if positions.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"positions must be int32 or int64, not {positions.dtype}")
    if positions.shape[0] != tokens:
        raise ValueError(f"positions needs {tokens} entries, not {positions.shape[0]}")
    return (positions.data_ptr(), positions.element_size(), freqs.data_ptr(), freqs.shape[0])


def rotary_frequencies(dim: int, base: float = 10000.0, scaling: str = "none",
                       factor: float = 1.0, original: float = 4096.0, device=None):
    """lssvm_rotary_frequencies: (frequencies, scale) of the rotary positions of `dim`
    values of a head (even), for ``rotary`` and ``cache_append``.

    scaling stretches them by `factor` for contexts longer than trained ones: "linear"
    divides every frequency, "ntk" raises the base so that the slowest pair is
    stretched by factor and the fastest kept, "yarn" keeps the pairs that turn 32 times
    or more over `original` positions, divides those of one turn or fewer, mixes
    between, and gives a scale of 0.1 ln(factor) + 1."""
    torch = _torch()
    if scaling not in SCALINGS:
        raise ValueError(f"unknown scaling {scaling!r}")
    if dim < 2 or dim % 2:
        raise ValueError("dim must be even and positive")
    freqs = torch.empty(dim // 2, dtype=torch.float64)
    scale = _D(0.0)
    _check(_lib().lssvm_rotary_frequencies(
        dim // 2, float(base), SCALINGS[scaling], float(factor), float(original),
        ctypes.cast(freqs.data_ptr(), ctypes.POINTER(_D)), ctypes.byref(scale)))
    return (freqs if device is None else freqs.to(device)), scale.value


def rotary(x, positions, freqs, scale: float = 1.0, interleaved: bool = False,
           transpose: bool = False, out=None):
    """lssvm_rotary: the heads of x (tokens x heads x dim) turned by their positions.

    The first 2 * len(freqs) values of a head are turned, pair (2i, 2i + 1) if
    interleaved, else (i, i + len(freqs)), and multiplied by scale; the others are
    copied. transpose applies the transposed map, which is the gradient's. out may be
    x itself."""
    torch = _torch()
    _gpu(x, "x", 3)
    code = _code(x.dtype)
    if out is None:
        out = torch.empty_like(x)
    else:
        _gpu(out, "out", 3, x.dtype, x.device)
        if out.shape != x.shape:
            raise ValueError(f"out must have the shape of x, {tuple(x.shape)}")
        _no_gradient(out.requires_grad)
    _no_gradient(x.requires_grad)
    tokens, heads, dim = x.shape
    _call(x.device, _lib().lssvm_rotary, x.data_ptr(), _two(*x.stride()), out.data_ptr(),
          _two(*out.stride()), tokens, heads, dim,
          *_angles(positions, freqs, tokens, x.device), scale, interleaved, transpose, code)
    return out


def cache_append(cache, k, v, offsets, positions=None, freqs=None, scale: float = 1.0,
                 interleaved: bool = False) -> None:
    """lssvm_cache_append: writes new tokens (tokens x heads x dim) into the cache.

    Sequence s gets the tokens offsets[s] .. offsets[s + 1] - 1 as its last keys, which
    cache.lengths already counts. With freqs, keys are turned by their positions on the
    way (``rotary``). Weights of the new keys become zero."""
    _cache(cache)
    _rows(k, "k", cache, cache.heads)
    _rows(v, "v", cache, cache.heads)
    tokens = k.shape[0]
    if v.shape[0] != tokens:
        raise ValueError("k and v must have the same tokens")
    if (positions is None) != (freqs is None):
        raise ValueError("positions and freqs are given together")
    _no_gradient(k.requires_grad or v.requires_grad or cache.k.requires_grad or
                 cache.v.requires_grad)
    angles = (None, 0, None, 0) if freqs is None else _angles(positions, freqs, tokens,
                                                              cache.device)
    _call(cache.device, _lib().lssvm_cache_append, cache._ref, k.data_ptr(), _two(*k.stride()),
          v.data_ptr(), _two(*v.stride()), tokens, _offsets(offsets, cache), *angles, scale,
          interleaved)


def attention_workspace_bytes(cache, tokens: int, heads: int, accumulate: bool = False) -> int:
    """lssvm_attention_workspace_bytes: workspace of ``attention`` for that many rows."""
    return int(_lib().lssvm_attention_workspace_bytes(_cache(cache)._ref, tokens, heads,
                                                      accumulate))


def attention(q, cache, offsets, scale: float | None = None, causal: bool = True,
              accumulate: bool = False, weight_out=None, out=None, workspace=None):
    """lssvm_attention: rows q (tokens x heads x dim) over the cache.

    Sequence s has the rows offsets[s] .. offsets[s + 1] - 1. With causal they are its
    last tokens, and each sees the keys up to its own; else every key. scale is
    dim ** -0.5 if None. accumulate adds to each key's weight what the rows gave it:
    into weight_out (shaped as cache.weight) or, if None, into cache.weight itself.
    Rows outside the offsets are left as they were in out (not set in a new one)."""
    torch = _torch()
    _cache(cache)
    _rows(q, "q", cache)
    tokens, heads, dim = q.shape
    if out is None:
        out = torch.empty_like(q)
    else:
        _rows(out, "out", cache, heads)
        if out.shape[0] != tokens:
            raise ValueError(f"out must have the shape of q, {tuple(q.shape)}")
        _no_gradient(out.requires_grad)
    _no_gradient(q.requires_grad or cache.k.requires_grad or cache.v.requires_grad)
    w = None
    if weight_out is not None:
        if not accumulate:
            raise ValueError("weight_out needs accumulate")
        _gpu(weight_out, "weight_out", 3, torch.float32, cache.device)
        if weight_out.shape != cache.k.shape[:3]:
            raise ValueError(f"weight_out must be {tuple(cache.k.shape[:3])}")
        w = weight_out.stride()[:2]
    if workspace is None:
        workspace = alloc_workspace(attention_workspace_bytes(cache, tokens, heads, accumulate),
                                    cache.device)
    else:
        _workspace(workspace, cache.device)
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
    _call(cache.device, _lib().lssvm_attention, cache._ref, q.data_ptr(), _two(*q.stride()),
          tokens, heads, _offsets(offsets, cache), dim ** -0.5 if scale is None else scale, causal,
          accumulate, weight_out.data_ptr() if w else None, _two(*w) if w else None,
          out.data_ptr(), _two(*out.stride()), workspace.data_ptr(),
          workspace.numel() * workspace.element_size())
    return out


def cache_evict(cache, target, budget: int, recent: int = 0, kept=None):
    """lssvm_cache_evict: copies the keys that stay into the pages of `target`: of every
    sequence and head the last `recent` and the heaviest of the others, `budget` in
    all. Returns the kept indices (sequences x heads x budget, int32, rising, then -1);
    target.lengths becomes min(length, budget)."""
    torch = _torch()
    _cache(cache)
    _cache(target, "target")
    if target.device != cache.device:
        raise ValueError(f"target must be on {cache.device}, not {target.device}")
    _no_gradient(any(t.requires_grad for c in (cache, target) for t in (c.k, c.v)))
    shape = (cache.sequences, cache.heads, budget)
    if kept is None:
        kept = torch.empty(shape, dtype=torch.int32, device=cache.device) if budget > 0 else None
    else:
        _gpu(kept, "kept", 3, torch.int32, cache.device)
        if tuple(kept.shape) != shape or not kept.is_contiguous():
            raise ValueError(f"kept must be {shape} and contiguous")
    _call(cache.device, _lib().lssvm_cache_evict, cache._ref, target._ref, budget, recent,
          kept.data_ptr() if kept is not None else None)
    return kept
