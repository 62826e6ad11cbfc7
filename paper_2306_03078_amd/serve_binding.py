"""ctypes binding of the entry points around a decode step's attention (include/spqr_serve.h): argument marshalling only.

A SpQRStep holds the device arrays of a step and the descriptor that points into them; every computation runs in the
library's kernels.  No CPU fallback: a missing libspqr.so raises.
"""
from __future__ import annotations

import ctypes as C
import math

from . import binding as B
from .binding import SPQR_F16, SPQR_F32, SpQRError, load_library

SPQR_BF16 = 2
SPQR_MAX_REQUESTS, SPQR_MAX_FRESH = 1024, 256


class spqr_step_t(C.Structure):
    _fields_ = ([(k, C.c_int32) for k in ("requests", "tokens", "max_fresh", "max_pages", "mask_words", "dtype", "heads", "kv_heads",
                                          "head_dim", "page", "pages", "layers", "rotary_dim", "rotary_positions", "rotary_pairs")]
                + [("scale", C.c_float)]
                + [(k, C.c_void_p) for k in ("k", "v", "cached", "fresh", "held", "table", "parent", "pool", "ends", "q_start",
                                             "position", "slot", "mask", "held_out", "ends_out", "cached_out", "rotary", "workspace")]
                + [("workspace_bytes", C.c_int64)])


class spqr_rows_t(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("q", "k", "v")] + [(k, C.c_int64) for k in ("q_stride", "k_stride", "v_stride")] + \
               [("x_dtype", C.c_int32)]


_entry = {}
_dtypes = {}
_current_device = _raw_stream = _int32 = None       # torch's, where this torch has the raw calls (see binding._stream_ptr)


def _lib():
    global _current_device, _raw_stream, _int32
    lib = load_library()
    if not _entry:
        import torch
        S, R, i32, i64, vp = C.POINTER(spqr_step_t), C.c_void_p, C.c_int32, C.c_int64, C.c_void_p
        for name, rest in (("spqr_cache_plan", [vp]), ("spqr_cache_store", [i32, R, vp, vp]),
                           ("spqr_tree_attention", [i32, vp, i64, vp, i64, vp]), ("spqr_cache_keep", [vp, vp])):
            f = getattr(lib, name)
            f.restype, f.argtypes = C.c_int, [S] + rest
            _entry[name] = f if B._call is B._ctypes_call else C.cast(f, C.c_void_p).value
        lib.spqr_tree_attention_workspace_bytes.restype = i64
        lib.spqr_tree_attention_workspace_bytes.argtypes = [S]
        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)
        _int32 = torch.int32
        _dtypes.update({torch.float32: SPQR_F32, torch.float16: SPQR_F16, torch.bfloat16: SPQR_BF16})
    return lib


def _run(name, step, stream, *args):
    """One of the entries, on the step's device: launches go to the current one, on its current stream where none is given."""
    if _current_device() != step._index:
        import torch
        with torch.cuda.device(step._index):
            return _run(name, step, stream, *args)
    rc = B._call(_entry[name], step.desc, *args, _raw_stream(step._index) if stream is None else stream.cuda_stream)
    if rc != 0:
        raise SpQRError(int(rc), name)


# the arrays of a descriptor: their type, and their shape in terms of the step's sizes
_ARRAYS = {
    "cached": ("int32", lambda s: (s.requests,)), "fresh": ("int32", lambda s: (s.requests,)), "held": ("int32", lambda s: (s.requests,)),
    "table": ("int32", lambda s: (s.requests, s.max_pages)), "parent": ("int32", lambda s: (s.tokens,)),
    "pool": ("int32", lambda s: (s.pages,)), "ends": ("int64", lambda s: (3,)), "q_start": ("int32", lambda s: (s.requests + 1,)),
    "position": ("int32", lambda s: (s.tokens,)), "slot": ("int32", lambda s: (s.tokens,)),
    "mask": ("int64", lambda s: (s.tokens, s.mask_words)), "held_out": ("int32", lambda s: (s.requests,)),
    "ends_out": ("int64", lambda s: (3,)), "cached_out": ("int32", lambda s: (s.requests,)),
}


class SpQRStep:
    """The arrays of a decode step over a paged cache, and the descriptor of them.

    k_cache, v_cache: [layers, pages, kv_heads, page, head_dim] float16 or bfloat16 device tensors (None for a step that
    is only planned: give page and pages).  heads: query heads.  requests, tokens, max_pages: sizes, where no array given says
    them.  Any array of include/spqr_serve.h can be given by its name; the others are made here: empty requests, and an
    empty table with a ring that has all pages (pool and ends are only made with a table).  parent (int32 [tokens]) is None
    unless given, mask exists where mask_words > 0 or it is given.  rotary: float32 [positions, rotary_dim], cosines, then
    sines, or None.  scale: head_dim ** -0.5 if None.
    The step keeps the tensors alive and owns the attention's scratch: use it on one stream at a time (the first call may be on any: what the
    constructor does is done when it returns)."""

    def __init__(self, k_cache, v_cache, heads=1, *, requests=None, tokens=None, max_pages=None, page=None, pages=None, mask_words=None,
                 rotary=None, rotary_pairs=False, scale=None, max_fresh=0, device="cuda", **arrays):
        import torch
        lib = _lib()
        unknown = set(arrays) - set(_ARRAYS)
        if unknown:
            raise TypeError(f"no array of a step: {', '.join(sorted(unknown))}")
        given = {n: a for n, a in arrays.items() if a is not None}
        if (k_cache is None) != (v_cache is None):
            raise ValueError("k_cache and v_cache: both or neither")
        d = self.desc = spqr_step_t()
        d.layers = d.kv_heads = 1
        d.head_dim, d.dtype, self.dtype = 64, SPQR_F16, torch.float16
        if k_cache is not None:
            if (k_cache.dim() != 5 or k_cache.shape != v_cache.shape or k_cache.dtype != v_cache.dtype or k_cache.device != v_cache.device
                    or k_cache.dtype not in (torch.float16, torch.bfloat16) or not k_cache.is_contiguous() or not v_cache.is_contiguous()
                    or not k_cache.is_cuda):
                raise ValueError("k_cache, v_cache: contiguous float16 or bfloat16 device tensors [layers, pages, kv_heads, page, head_dim]")
            device, self.dtype, d.dtype = k_cache.device, k_cache.dtype, _dtypes[k_cache.dtype]
            d.layers, d.pages, d.kv_heads, d.page, d.head_dim = k_cache.shape
            if page not in (None, d.page) or pages not in (None, d.pages):
                raise ValueError(f"the cache has {d.pages} pages of {d.page} rows")
            d.k, d.v = k_cache.data_ptr(), v_cache.data_ptr()
        elif page is None or pages is None:
            raise ValueError("a step without caches: page and pages as numbers")
        else:
            d.page, d.pages = page, pages
        self.k_cache, self.v_cache = k_cache, v_cache
        self.requests, self.tokens, self.max_pages, self.mask_words = requests, tokens, max_pages, mask_words
        self.page, self.pages, self.heads, self.kv_heads, self.head_dim = d.page, d.pages, int(heads), d.kv_heads, d.head_dim
        for size, names, axis in (("requests", ("cached", "fresh", "held", "table"), 0), ("max_pages", ("table",), 1),
                                  ("tokens", ("slot", "position", "parent", "mask"), 0), ("mask_words", ("mask",), 1)):
            for n in names:
                if getattr(self, size) is None and n in given:
                    setattr(self, size, given[n].shape[axis])
        if self.mask_words is None:
            self.mask_words = 0
        if None in (self.requests, self.tokens, self.max_pages):
            raise ValueError("requests, tokens and max_pages: as numbers, or by an array of their size")
        d.requests, d.tokens, d.max_pages, d.mask_words = self.requests, self.tokens, self.max_pages, self.mask_words
        d.heads, d.max_fresh, d.rotary_pairs = self.heads, int(max_fresh), int(bool(rotary_pairs))
        d.scale = float(scale) if scale is not None else 1.0 / math.sqrt(d.head_dim)
        if not math.isfinite(d.scale):
            raise ValueError(f"scale: a finite number, not {scale}")
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError(f"a step's arrays are in device memory, not on {self.device}")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index

        def on_device(a):
            return a.device == self.device

        # the arrays that are not given, in one buffer
        missing = [n for n in _ARRAYS if n not in given and n != "parent" and (n != "mask" or self.mask_words)
                   and (n not in ("pool", "ends") or "table" not in given)]
        sizes = [math.prod(_ARRAYS[n][1](self)) * (2 if _ARRAYS[n][0] == "int64" else 1) for n in missing]
        places = [0]
        for k in sizes:
            places.append(places[-1] + -(-k // 64) * 64)
        buffer = torch.zeros(places[-1], dtype=torch.int32, device=self.device)
        for n, k, at in zip(missing, sizes, places):
            dtype, shape = _ARRAYS[n]
            given[n] = buffer[at:at + k].view(getattr(torch, dtype)).view(shape(self))
        if "table" in missing:
            given["table"].fill_(-1)
        if "pool" in missing:
            torch.arange(self.pages, dtype=torch.int32, device=self.device, out=given["pool"])
        if "ends" in missing:
            given["ends"][1] = self.pages
        for n, (dtype, shape) in _ARRAYS.items():
            a = given.get(n)
            if a is not None:
                if a.dtype != getattr(torch, dtype) or not a.is_contiguous() or tuple(a.shape) != shape(self) or not on_device(a):
                    raise ValueError(f"{n}: a contiguous {dtype} tensor {list(shape(self))} on {self.device}, not {a.dtype} {list(a.shape)} on {a.device}")
                setattr(d, n, a.data_ptr())
            setattr(self, n, a)
        self.rotary = rotary
        if rotary is not None:
            if rotary.dtype != torch.float32 or rotary.dim() != 2 or not rotary.is_contiguous() or not on_device(rotary):
                raise ValueError("rotary: a contiguous float32 device tensor [positions, rotary_dim]")
            d.rotary, d.rotary_positions, d.rotary_dim = rotary.data_ptr(), rotary.shape[0], rotary.shape[1]
        self.workspace = None
        if k_cache is not None:
            need = int(lib.spqr_tree_attention_workspace_bytes(C.byref(d)))
            if need < 0:
                raise SpQRError(need, "spqr_tree_attention_workspace_bytes")
            self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
            d.workspace, d.workspace_bytes = self.workspace.data_ptr(), self.workspace.numel()
        T, D = self.tokens, self.head_dim
        self._q_like, self._kv_like = (((T, h, D), (h * D, D, 1), self._index) for h in (self.heads, self.kv_heads))
        self._q_of = torch.empty(1, dtype=self.dtype, device=self.device).expand(T, self.heads, D)
        self._rows = spqr_rows_t()
        self._rows_at = C.addressof(self._rows)
        B._wait_for(self.device)

    def advance(self):
        """The next step's lengths and pages are this one's results: cached and cached_out, held and held_out, ends and
        ends_out change places (pointers only; a step captured in a graph keeps the ones it was captured with)."""
        for a, b in (("cached", "cached_out"), ("held", "held_out"), ("ends", "ends_out")):
            x, y = getattr(self, a), getattr(self, b)
            setattr(self, a, y)
            setattr(self, b, x)
            setattr(self.desc, a, y.data_ptr())
            setattr(self.desc, b, x.data_ptr())


def spqr_cache_plan(step: SpQRStep, stream=None) -> SpQRStep:
    """Pages, slots, positions and masks of a step's new tokens: fills table, q_start, slot, position, mask, held_out, ends_out."""
    _run("spqr_cache_plan", step, stream)
    return step


def _row_stride(x, like, name):
    """Elements between the rows of x: [tokens, heads, head_dim] or [tokens, heads * head_dim], each row contiguous.  like: the
    shape and strides of the dense one, and the device's index."""
    if x.get_device() != like[2]:
        raise ValueError(f"{name}: a tensor on cuda:{like[2]}, not on {x.device}")
    shape, strides = x.shape, x.stride()
    if shape == like[0] and strides == like[1]:
        return strides[0]
    (tokens, heads, head_dim), row = like[0], like[1][0]
    if len(shape) == 3:
        fits = shape == like[0] and strides[2] == 1 and (heads == 1 or strides[1] == head_dim)
    else:
        fits = shape == (tokens, row) and strides[1] == 1
    if not fits:
        raise ValueError(f"{name}: [{tokens}, {heads}, {head_dim}] with contiguous rows, not {list(shape)} with strides {list(strides)}")
    return strides[0] if tokens > 1 else row


def spqr_cache_store(step: SpQRStep, q, k, v, layer: int = 0, out=None, stream=None):
    """q turned by its rows' positions (a tensor of the cache's type [tokens, heads, head_dim], returned); k turned, and v,
    stored in their slots of `layer`.  q, k, v: float32, float16 or bfloat16, rows of one step's products."""
    if stream is not None and out is None:
        with B._on(stream):
            return spqr_cache_store(step, q, k, v, layer, out)
    x = step._rows
    dtype = q.dtype
    if dtype not in _dtypes or k.dtype != dtype or v.dtype != dtype:
        raise ValueError(f"q, k, v: one type of float32, float16, bfloat16, not {q.dtype}, {k.dtype}, {v.dtype}")
    x.q_stride = _row_stride(q, step._q_like, "q")
    x.k_stride = _row_stride(k, step._kv_like, "k")
    x.v_stride = _row_stride(v, step._kv_like, "v")
    x.q, x.k, x.v, x.x_dtype = q.data_ptr(), k.data_ptr(), v.data_ptr(), _dtypes[dtype]
    if out is None:
        import torch
        out = torch.empty_like(step._q_of, memory_format=torch.contiguous_format)
    elif out.dtype != step.dtype or not out.is_contiguous() or out.numel() != step._q_of.numel() or out.get_device() != step._index:
        raise ValueError(f"out: a contiguous {step.dtype} tensor {list(step._q_like[0])} on {step.device}")
    _run("spqr_cache_store", step, stream, layer, step._rows_at, out)
    return out


def spqr_tree_attention(step: SpQRStep, q, layer: int = 0, out=None, stream=None):
    """Attention of the step's rows q [tokens, heads, head_dim] (the cache's type) over the cached tokens of their requests and
    the new ones that their masks show; out has q's shape (rows that belong to no request are left as they are)."""
    if stream is not None and out is None:
        with B._on(stream):
            return spqr_tree_attention(step, q, layer, out)
    if q.dtype != step.dtype:
        raise ValueError(f"q: {step.dtype}, not {q.dtype}")
    q_stride = _row_stride(q, step._q_like, "q")
    if out is None:
        import torch
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        out_stride = step._q_like[1][0]
    else:
        if out.dtype != step.dtype:
            raise ValueError(f"out: {step.dtype}, not {out.dtype}")
        out_stride = _row_stride(out, step._q_like, "out")
    _run("spqr_tree_attention", step, stream, layer, q, q_stride, out, out_stride)
    return out


def spqr_cache_keep(step: SpQRStep, last=None, stream=None):
    """After verification: last [requests] int32, the last accepted new token of each request (-1: none), or None: all.  The
    accepted rows move together in all layers; returns step.cached_out, the new lengths (up to the first token that was not stored:
    where pages were lacking, the lengths grow by less than the path)."""
    if last is not None and (last.dtype != _int32 or not last.is_contiguous() or last.numel() != step.requests
                             or last.get_device() != step._index):
        raise ValueError(f"last: a contiguous int32 tensor [{step.requests}] on {step.device}")
    _run("spqr_cache_keep", step, stream, last)
    return step.cached_out
