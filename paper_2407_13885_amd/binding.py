"""Thin ctypes binding of ``libattnw.so`` -- argument marshalling only.

Every step of the path (contraction, scaling, row max, exponentials, row sum,
normalisation, stores) runs inside the HIP kernels behind the C ABI declared
in ``include/attnw.h``.  The functions here have the same names as the C entry
points, accept either raw device addresses (ints) or objects with a
``data_ptr()`` method (PyTorch tensors), and raise :class:`AttnwError` on a
non-zero status.  There is no CPU fallback: a missing library is an error.

A small call costs the host more than the device, so the public functions pass
their arguments on to callables of ``_entry.so`` (``csrc/entry.cpp``), which hand
the usual kinds straight to the C function and everything else to the functions
written here.
"""
from __future__ import annotations

import ctypes
import functools
import importlib
import inspect
import os
import subprocess
import sysconfig
import warnings
from typing import Optional

ATTNW_F32 = 0
ATTNW_BF16 = 1
ATTNW_HALVES = 0
ATTNW_PAIRS = 1
ATTNW_SECTIONS = 0
ATTNW_TURNS = 1

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
_CSRC = os.path.join(_PKG, "csrc")
_LIB = os.path.join(_PKG, "libattnw.so")
_ENTRY = os.path.join(_PKG, "_entry.so")

EXPORTS = ("attnw_fused", "attnw_softmax", "attnw_softmax_cast", "attnw_gemm_scores", "attnw_scale", "attnw_attention",
           "attnw_rotary_table", "attnw_rotary", "attnw_cache_append", "attnw_paged_workspace", "attnw_paged_attention",
           "attnw_paged_sums", "attnw_cache_evict", "attnw_rotary_axes_table", "attnw_rotary_axes", "attnw_byte_cache_append", "attnw_byte_paged_workspace",
           "attnw_byte_paged_attention", "attnw_status_string", "attnw_version")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]

_lib = None
_entry = None
_entries = {}               # the public functions by name
_points = []                # (function that one stands for, kinds of its arguments, what it looks `direct` up in)
_direct = {}                # the callables of _entry.so among what they call
_word_points = []           # the same for entry points of addresses and whole numbers in any order
_word_direct = {}


class AttnwError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libattnw status {status}: {message}")
        self.status = status


def library_path() -> str:
    return _LIB


def sources() -> list:
    return sorted(os.path.join(_CSRC, f) for f in os.listdir(_CSRC) if f.endswith(".hip"))


def build(verbose: bool = False) -> str:
    """Compile every HIP source for gfx950 into ``libattnw.so`` (always recompiles): one hipcc process per
    source, side by side, objects in a temporary directory, then one link step; and ``_entry.so``."""
    import concurrent.futures
    import shutil
    import tempfile
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    include = ["-I", os.path.join(_ROOT, "include"), "-I", _CSRC]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        proc = subprocess.run(cmd, capture_output=True, text=True)
        if proc.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + " ".join(cmd) + "\n" + proc.stdout + proc.stderr)

    with tempfile.TemporaryDirectory(prefix="attnw_build_") as tmp:
        entry = os.path.join(tmp, "_entry.so")
        run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-Wall", "-Wno-missing-field-initializers", "-shared", "-fPIC", "-I",
             sysconfig.get_paths()["include"], os.path.join(_CSRC, "entry.cpp"), "-o", entry])
        shutil.move(entry, _ENTRY)                # (a new file: a process that has loaded the old one keeps it)
        jobs = [(src, os.path.join(tmp, os.path.basename(src) + ".o")) for src in sources()]
        workers = max(1, min(len(jobs), os.cpu_count() or 1, 8))
        with concurrent.futures.ThreadPoolExecutor(max_workers=workers) as pool:
            list(pool.map(lambda j: run([hipcc, *compile_flags, *include, "-c", j[0], "-o", j[1]]), jobs))
        run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *[o for _, o in jobs], "-o", _LIB])
    global _lib
    _lib = None
    for entry in [*_direct.values(), *_word_direct.values()]:     # (their C functions are the old library's)
        entry.bind(0)
    _attach()
    return _LIB


def load_library():
    """Load ``libattnw.so``; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB):
            raise FileNotFoundError(
                f"{_LIB} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
        lib = ctypes.CDLL(_LIB)
        i64, vp, ci, cf = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float
        lib.attnw_fused.argtypes = [vp, vp, vp, i64, i64, i64, i64, cf, ci, vp]
        lib.attnw_fused.restype = ci
        lib.attnw_gemm_scores.argtypes = [vp, vp, vp, i64, i64, i64, i64, cf, ci, vp]
        lib.attnw_gemm_scores.restype = ci
        lib.attnw_attention.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, cf, ci, vp]
        lib.attnw_attention.restype = ci
        lib.attnw_softmax.argtypes = [vp, vp, i64, i64, ci, vp]
        lib.attnw_softmax.restype = ci
        lib.attnw_softmax_cast.argtypes = [vp, vp, i64, i64, ci, ci, vp]
        lib.attnw_softmax_cast.restype = ci
        lib.attnw_scale.argtypes = [vp, vp, i64, ctypes.c_float, ci, vp]
        lib.attnw_scale.restype = ci
        cd = ctypes.c_double
        lib.attnw_rotary_table.argtypes = [vp, i64, i64, cd, cd, cd, cd, cd, cd, vp]
        lib.attnw_rotary.argtypes = [vp] * 4 + [i64] * 7 + [ci] * 3 + [vp]
        lib.attnw_cache_append.argtypes = [vp] * 8 + [i64] * 6 + [ci, vp]
        lib.attnw_paged_workspace.argtypes = [vp, i64, i64]
        lib.attnw_paged_attention.argtypes = [vp] * 6 + [i64] * 3 + [vp, i64, vp]
        lib.attnw_paged_sums.argtypes = [vp] * 7 + [i64] * 3 + [vp]
        lib.attnw_cache_evict.argtypes = [vp] * 5 + [i64] * 2 + [vp]
        lib.attnw_rotary_axes_table.argtypes = [vp, vp, i64, i64, cd, cd, cd, cd, cd, cd, vp]
        lib.attnw_rotary_axes.argtypes = [vp] * 5 + [i64] * 7 + [ci] * 3 + [vp]
        lib.attnw_byte_cache_append.argtypes = [vp] * 9 + [i64] * 6 + [ci, vp]
        lib.attnw_byte_paged_workspace.argtypes = [vp, i64, i64]
        lib.attnw_byte_paged_attention.argtypes = [vp] * 6 + [i64] * 3 + [vp, i64, vp]
        for name in ("rotary_table", "rotary", "cache_append", "paged_attention", "paged_sums", "cache_evict", "rotary_axes_table", "rotary_axes", "byte_cache_append",
                     "byte_paged_attention"):
            getattr(lib, f"attnw_{name}").restype = ci
        lib.attnw_paged_workspace.restype = i64
        lib.attnw_byte_paged_workspace.restype = i64
        lib.attnw_status_string.argtypes = [ci]
        lib.attnw_status_string.restype = ctypes.c_char_p
        lib.attnw_version.argtypes = []
        lib.attnw_version.restype = ci
        _lib = lib
        for name, entry in [*_direct.items(), *_word_direct.items()]:
            entry.bind(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value)
    return _lib


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr())
    return int(x)


def _struct(x, kind) -> Optional[int]:
    if x is None:
        return None
    if not isinstance(x, kind):                   # (the host reads it: an address of anything else would crash the process)
        raise TypeError(f"{kind.__name__} expected, not {type(x).__name__}")
    return x._address


def _stream(stream) -> Optional[int]:
    if stream is None:
        return None
    if hasattr(stream, "cuda_stream"):      # torch.cuda.Stream exposes the hipStream_t here
        return int(stream.cuda_stream)
    return int(stream)


def _check(status: int) -> None:
    if status != 0:
        raise AttnwError(status, attnw_status_string(status))


def attnw_status_string(status: int) -> str:
    return load_library().attnw_status_string(int(status)).decode()


def attnw_version() -> int:
    return int(load_library().attnw_version())


def _in_front(function, points, kinds):
    """A function of the same signature that calls what its scope has as `direct`: `function`, until _attach puts a callable of ``_entry.so`` there."""
    name, arguments = function.__name__, ", ".join(inspect.signature(function).parameters)
    scope = {"direct": function}
    exec(f"def {name}({arguments}):\n    return direct({arguments})", scope)
    points.append((function, kinds, scope))
    _entries[name] = functools.update_wrapper(scope[name], function)
    _entries[name].__defaults__ = function.__defaults__
    return _entries[name]


def _entry_point(pointers: int, sizes: int, scales: int, dtypes: int):
    """The function by way of a callable of ``_entry.so``, for arguments: pointers, sizes, a scale, element types, a stream.  What
    is returned is a function still, of the same signature (copied, pickled, referred to weakly, inspected, bound like one)."""
    return lambda function: _in_front(function, _points, (pointers, sizes, scales, dtypes))


def _word_entry_point(kinds: str, *structures):
    """The same for arguments of the given kinds (s: a structure, of the next of the types, p: an address, i: a whole number, n: one of 32 bits)
    and a stream."""
    return lambda function: _in_front(function, _word_points, (kinds, structures))


def _attach() -> None:
    """The public functions onto ``_entry.so``, once it is there; ctypes alone until then, and aloud if it is there and does not load."""
    global _entry
    if _entry is not None or not os.path.exists(_ENTRY):
        return
    try:
        importlib.invalidate_caches()
        _entry = importlib.import_module("._entry", __package__)
    except ImportError as e:
        warnings.warn(f"{_ENTRY} does not load, calls take the longer way through ctypes: {e}", RuntimeWarning, stacklevel=2)
        return
    for function, kinds, scope in _points:
        scope["direct"] = _direct[function.__name__] = _entry.Entry(function, _check, *kinds)
    try:
        entries = [_entry.Words(function, _check, *kinds) for function, kinds, _ in _word_points]
    except (AttributeError, TypeError, ValueError):   # (built from sources older than this file: ctypes alone for these until the next build)
        return
    for (function, _, scope), entry in zip(_word_points, entries):
        scope["direct"] = _word_direct[function.__name__] = entry


@_entry_point(3, 4, 1, 1)
def attnw_fused(Q, K, P, B: int, H: int, N: int, d: int, scale: float, dtype: int, stream=None) -> None:
    """P = softmax(scale * Q K^T) over keys; see ``attnw_fused`` in include/attnw.h."""
    _check(load_library().attnw_fused(_ptr(Q), _ptr(K), _ptr(P), B, H, N, d, float(scale), int(dtype),
                                      _stream(stream)))


@_entry_point(2, 2, 0, 1)
def attnw_softmax(S, P, rows: int, cols: int, dtype: int, stream=None) -> None:
    """Row softmax of S into P; see ``attnw_softmax`` in include/attnw.h."""
    _check(load_library().attnw_softmax(_ptr(S), _ptr(P), rows, cols, int(dtype), _stream(stream)))


@_entry_point(2, 2, 0, 2)
def attnw_softmax_cast(S, P, rows: int, cols: int, in_dtype: int, out_dtype: int, stream=None) -> None:
    """Row softmax with separate input and output types; see ``attnw_softmax_cast`` in include/attnw.h."""
    _check(load_library().attnw_softmax_cast(_ptr(S), _ptr(P), rows, cols, int(in_dtype), int(out_dtype),
                                             _stream(stream)))


@_entry_point(2, 1, 1, 1)
def attnw_scale(X, Y, count: int, scale: float, dtype: int, stream=None) -> None:
    """Y = scale * X elementwise; see ``attnw_scale`` in include/attnw.h."""
    _check(load_library().attnw_scale(_ptr(X), _ptr(Y), count, float(scale), int(dtype), _stream(stream)))


@_entry_point(3, 4, 1, 1)
def attnw_gemm_scores(Q, K, S, B: int, H: int, N: int, d: int, scale: float, dtype: int, stream=None) -> None:
    """S = scale * Q K^T written to device memory; see ``attnw_gemm_scores`` in include/attnw.h."""
    _check(load_library().attnw_gemm_scores(_ptr(Q), _ptr(K), _ptr(S), B, H, N, d, float(scale), int(dtype),
                                            _stream(stream)))


@_entry_point(4, 4, 1, 1)
def attnw_attention(Q, K, V, O, B: int, H: int, N: int, d: int, scale: float, dtype: int, stream=None) -> None:
    """O = softmax(scale * Q K^T) V, weights kept on chip; see ``attnw_attention`` in include/attnw.h."""
    _check(load_library().attnw_attention(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), B, H, N, d, float(scale), int(dtype),
                                          _stream(stream)))


class AttnwCache(ctypes.Structure):
    """A paged cache; see ``attnw_cache`` in include/attnw.h.  K, V, table and lengths: addresses or tensors, which it keeps alive."""
    _fields_ = [("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("batch", ctypes.c_int64), ("pages", ctypes.c_int64), ("max_pages", ctypes.c_int64), ("page_size", ctypes.c_int64),
                ("kv_heads", ctypes.c_int64), ("d", ctypes.c_int64), ("dtype", ctypes.c_int32)]

    def __init__(self, K, V, table, lengths, batch: int, pages: int, max_pages: int, page_size: int, kv_heads: int, d: int, dtype: int):
        super().__init__(_ptr(K), _ptr(V), _ptr(table), _ptr(lengths), batch, pages, max_pages, page_size, kv_heads, d, dtype)
        self._kept = (K, V, table, lengths)
        self._address = ctypes.addressof(self)


class AttnwRule(ctypes.Structure):
    """What scores are made of beside the products, and what a token sees; see ``attnw_rule`` in include/attnw.h."""
    _fields_ = [("scale", ctypes.c_float), ("cap", ctypes.c_float), ("slopes", ctypes.c_void_p), ("prefix", ctypes.c_void_p),
                ("window", ctypes.c_int64)]

    def __init__(self, scale: float, cap: float = 0.0, slopes=None, prefix=None, window: int = 0):
        super().__init__(scale, cap, _ptr(slopes), _ptr(prefix), window)
        self._kept = (slopes, prefix)
        self._address = ctypes.addressof(self)


class AttnwAxes(ctypes.Structure):
    """Axes of rotary positions: how many pairs of columns each has; see ``attnw_axes`` in include/attnw.h."""
    _fields_ = [("count", ctypes.c_int32), ("order", ctypes.c_int32), ("fresh", ctypes.c_int32), ("pairs", ctypes.c_int32 * 4)]

    def __init__(self, pairs, order: int = ATTNW_SECTIONS, fresh: int = 0):
        pairs = tuple(pairs)
        super().__init__(len(pairs), int(order), int(fresh), (ctypes.c_int32 * 4)(*pairs[:4]))
        self._address = ctypes.addressof(self)


class AttnwByteCache(ctypes.Structure):
    """A paged cache in 8 bits; see ``attnw_byte_cache`` in include/attnw.h.  Addresses or tensors, which it keeps alive."""
    _fields_ = [("cache", AttnwCache), ("K_scales", ctypes.c_void_p), ("V_scales", ctypes.c_void_p), ("block", ctypes.c_int64)]

    def __init__(self, K, V, K_scales, V_scales, table, lengths, batch: int, pages: int, max_pages: int, page_size: int, block: int, kv_heads: int, d: int,
                 dtype: int):
        super().__init__(AttnwCache(K, V, table, lengths, batch, pages, max_pages, page_size, kv_heads, d, dtype), _ptr(K_scales), _ptr(V_scales), block)
        self._kept = (K, V, K_scales, V_scales, table, lengths)
        self._address = ctypes.addressof(self)


def _cache(x) -> Optional[int]:
    return _struct(x, AttnwCache)


def _rule(x) -> Optional[int]:
    return _struct(x, AttnwRule)


def _axes(x) -> Optional[int]:
    return _struct(x, AttnwAxes)


def _byte_cache(x) -> Optional[int]:
    return _struct(x, AttnwByteCache)


def attnw_rotary_table(table, positions: int, rot: int, base: float = 10000.0, factor: float = 1.0, low: float = 0.0,
                       high: float = 0.0, original: float = 0.0, gain: float = 1.0, stream=None) -> None:
    """Cosines and sines of rotary positions; see ``attnw_rotary_table`` in include/attnw.h."""
    _check(load_library().attnw_rotary_table(_ptr(table), positions, rot, base, factor, low, high, original, gain, _stream(stream)))


@_word_entry_point("ppppiiiiiiinnn")
def attnw_rotary(X, Y, table, positions, tokens: int, heads: int, d: int, rot: int, rows: int, x_stride: int, y_stride: int, layout: int,
                 inverse: int, dtype: int, stream=None) -> None:
    """Y = X with rotary positions, or the gradient of that; see ``attnw_rotary`` in include/attnw.h."""
    _check(load_library().attnw_rotary(_ptr(X), _ptr(Y), _ptr(table), _ptr(positions), tokens, heads, d, rot, rows, x_stride, y_stride,
                                       int(layout), int(inverse), int(dtype), _stream(stream)))


@_word_entry_point("spppppppiiiiiin", AttnwCache)
def attnw_cache_append(cache, Q, K, V, R, table, positions, starts, tokens: int, heads: int, rot: int, rows: int, q_stride: int,
                       kv_stride: int, layout: int, stream=None) -> None:
    """Queries turned, keys turned and values into the cache; see ``attnw_cache_append`` in include/attnw.h."""
    _check(load_library().attnw_cache_append(_cache(cache), _ptr(Q), _ptr(K), _ptr(V), _ptr(R), _ptr(table), _ptr(positions), _ptr(starts),
                                             tokens, heads, rot, rows, q_stride, kv_stride, int(layout), _stream(stream)))


def attnw_paged_workspace(cache, tokens: int, heads: int) -> int:
    """Bytes of workspace that ``attnw_paged_attention`` needs; see include/attnw.h."""
    size = int(load_library().attnw_paged_workspace(_cache(cache), tokens, heads))
    _check(min(size, 0))
    return size


@_word_entry_point("ssppppiiipi", AttnwCache, AttnwRule)
def attnw_paged_attention(cache, rule, Q, O, lse, starts, tokens: int, heads: int, q_stride: int, workspace, workspace_bytes: int,
                          stream=None) -> None:
    """Attention of new tokens over a paged cache; see ``attnw_paged_attention`` in include/attnw.h."""
    _check(load_library().attnw_paged_attention(_cache(cache), _rule(rule), _ptr(Q), _ptr(O), _ptr(lse), _ptr(starts), tokens, heads, q_stride,
                                                _ptr(workspace), workspace_bytes, _stream(stream)))


@_word_entry_point("sspppppiii", AttnwCache, AttnwRule)
def attnw_paged_sums(cache, rule, Q, lse, before, sums, starts, tokens: int, heads: int, q_stride: int, stream=None) -> None:
    """The weight that slots collect from new tokens; see ``attnw_paged_sums`` in include/attnw.h."""
    _check(load_library().attnw_paged_sums(_cache(cache), _rule(rule), _ptr(Q), _ptr(lse), _ptr(before), _ptr(sums), _ptr(starts), tokens, heads,
                                           q_stride, _stream(stream)))


@_word_entry_point("sspppii", AttnwCache, AttnwCache)
def attnw_cache_evict(cache, into, sums, into_sums, kept, keep: int, recent: int, stream=None) -> None:
    """The slots that collected the most weight into other pages; see ``attnw_cache_evict`` in include/attnw.h."""
    _check(load_library().attnw_cache_evict(_cache(cache), _cache(into), _ptr(sums), _ptr(into_sums), _ptr(kept), keep, recent, _stream(stream)))


def attnw_rotary_axes_table(table, axes, positions: int, rot: int, base: float = 10000.0, factor: float = 1.0, low: float = 0.0, high: float = 0.0,
                            original: float = 0.0, gain: float = 1.0, stream=None) -> None:
    """Cosines and sines of rotary positions with several axes; see ``attnw_rotary_axes_table`` in include/attnw.h."""
    _check(load_library().attnw_rotary_axes_table(_ptr(table), _axes(axes), positions, rot, base, factor, low, high, original, gain, _stream(stream)))


@_word_entry_point("ppppsiiiiiiinnn", AttnwAxes)
def attnw_rotary_axes(X, Y, table, positions, axes, tokens: int, heads: int, d: int, rot: int, rows: int, x_stride: int, y_stride: int, layout: int,
                      inverse: int, dtype: int, stream=None) -> None:
    """Y = X with rotary positions on several axes, or the gradient of that; see ``attnw_rotary_axes`` in include/attnw.h."""
    _check(load_library().attnw_rotary_axes(_ptr(X), _ptr(Y), _ptr(table), _ptr(positions), _axes(axes), tokens, heads, d, rot, rows, x_stride, y_stride,
                                            int(layout), int(inverse), int(dtype), _stream(stream)))


@_word_entry_point("sppppppspiiiiiin", AttnwByteCache, AttnwAxes)
def attnw_byte_cache_append(cache, Q, K, V, R, table, positions, axes, starts, tokens: int, heads: int, rot: int, rows: int, q_stride: int, kv_stride: int,
                        layout: int, stream=None) -> None:
    """Queries turned, keys turned and values into a cache in 8 bits; see ``attnw_byte_cache_append`` in include/attnw.h."""
    _check(load_library().attnw_byte_cache_append(_byte_cache(cache), _ptr(Q), _ptr(K), _ptr(V), _ptr(R), _ptr(table), _ptr(positions), _axes(axes), _ptr(starts),
                                              tokens, heads, rot, rows, q_stride, kv_stride, int(layout), _stream(stream)))


def attnw_byte_paged_workspace(cache, tokens: int, heads: int) -> int:
    """Bytes of workspace that ``attnw_byte_paged_attention`` needs; see include/attnw.h."""
    size = int(load_library().attnw_byte_paged_workspace(_byte_cache(cache), tokens, heads))
    _check(min(size, 0))
    return size


@_word_entry_point("ssppppiiipi", AttnwByteCache, AttnwRule)
def attnw_byte_paged_attention(cache, rule, Q, O, lse, starts, tokens: int, heads: int, q_stride: int, workspace, workspace_bytes: int, stream=None) -> None:
    """Attention of new tokens over a paged cache in 8 bits; see ``attnw_byte_paged_attention`` in include/attnw.h."""
    _check(load_library().attnw_byte_paged_attention(_byte_cache(cache), _rule(rule), _ptr(Q), _ptr(O), _ptr(lse), _ptr(starts), tokens, heads, q_stride,
                                                 _ptr(workspace), workspace_bytes, _stream(stream)))


_attach()
