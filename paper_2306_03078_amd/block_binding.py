"""ctypes binding of what a decoder's step does beside its products and its attention (include/spqr_block.h): argument marshalling only.

Each operator has a handle with what a program keeps from call to call (weights, sizes, scratch, small outputs); every computation
runs in the library's kernels.  No CPU fallback: a missing libspqr.so raises.  A handle is used on one stream at a time, and stays until
its last call has run; what its constructor does is done when it returns, so that the first call may be on any stream.  stream: that of
the call, None for the current one; tensors that a call makes are that stream's, as under torch.cuda.stream(stream); those that it is given are
ready there, and stay until it has run (Tensor.record_stream), as with torch's own calls.
"""
from __future__ import annotations

import ctypes as C
from struct import Struct

from . import binding as B
from . import serve_binding as S
from .binding import SpQRError, _wait_for
from .serve_binding import SPQR_MAX_REQUESTS

SPQR_MAX_WIDTH, SPQR_MAX_FUSED = 65536, 8
SPQR_ADAPTER_TILE, SPQR_MAX_SLOTS, SPQR_MAX_RANK, SPQR_MAX_ROWS = 64, 4096, 256, 1 << 20
SPQR_MAX_TOP = SPQR_MAX_GIVEN = 64
_NORMS = {None: 0, "rms": 1, "layer": 2}
_ACTS = {None: 0, "silu": 1, "sigmoid": 2, "tanh": 3}

_i32, _i64, _vp, _f32 = C.c_int32, C.c_int64, C.c_void_p, C.c_float


class spqr_residual_norm_t(C.Structure):
    _fields_ = ([(k, _i32) for k in ("rows", "width", "x_dtype", "y_dtype", "gate_dtype", "out_dtype", "weight_dtype", "norm_y", "norm_x", "act")]
                + [(k, _f32) for k in ("eps", "weight_offset", "skip", "scale")]
                + [(k, _vp) for k in ("x", "y", "gate", "sum", "out")]
                + [(k, _i64) for k in ("x_stride", "y_stride", "sum_stride", "out_stride", "gate_stride")]
                + [(k, _vp) for k in ("y_weight", "y_bias", "x_weight", "x_bias")])


class spqr_adapter_plan_t(C.Structure):
    _fields_ = [(k, _i32) for k in ("rows", "slots", "requests", "max_tiles")] + [(k, _vp) for k in ("adapter", "q_start", "count", "tile", "row")]


class spqr_adapters_t(C.Structure):
    _fields_ = ([(k, _i32) for k in ("count", "width", "slots", "dtype", "y_dtype")]
                + [(k, t * SPQR_MAX_FUSED) for k, t in (("m", _i32), ("max_rank", _i32), ("bank", _vp), ("scale", _vp), ("y", _vp),
                                                         ("out", _vp), ("y_stride", _i64), ("out_stride", _i64))]
                + [("x", _vp), ("x_stride", _i64), ("workspace", _vp), ("workspace_bytes", _i64)])


class spqr_token_logprobs_t(C.Structure):
    _fields_ = ([(k, _i32) for k in ("rows", "vocab", "dtype", "given", "top")] + [("scale", _f32), ("logits", _vp), ("stride", _i64)]
                + [(k, _vp) for k in ("tokens", "logprob", "entropy", "top_token", "top_logprob", "workspace")] + [("workspace_bytes", _i64)])


_entry = {}
_empty = _empty_like = _float32 = None                      # torch's
# What a call changes of a descriptor, written at once: a field at a time costs as much as the launch.
_norm_types, _norm_rows = Struct("=6i"), Struct("=10q")     # rows .. out_dtype (width among them); x .. out, x_stride .. gate_stride
_norm_rows_at = spqr_residual_norm_t.x.offset
_bank_rows, _bank_rows_at = Struct("=%dq" % (4 * SPQR_MAX_FUSED)), spqr_adapters_t.y.offset      # y, out, y_stride, out_stride


def _lib():
    global _empty, _empty_like, _float32
    lib = S._lib()
    if not _entry:
        import torch
        _empty, _empty_like, _float32 = torch.empty, torch.empty_like, torch.float32
        for name, rest in (("spqr_residual_norm", [_vp]), ("spqr_adapter_plan", [_vp]), ("spqr_adapters", [_vp, _vp]), ("spqr_token_logprobs", [_vp])):
            f = getattr(lib, name)
            f.restype, f.argtypes = C.c_int, [_vp] + rest
            _entry[name] = f if B._call is B._ctypes_call else C.cast(f, _vp).value
        lib.spqr_adapter_tiles.restype, lib.spqr_adapter_tiles.argtypes = _i32, [_i32, _i32]
        lib.spqr_adapters_bank_bytes.restype, lib.spqr_adapters_bank_bytes.argtypes = _i64, [_vp, _i32]
        lib.spqr_adapters_pack.restype, lib.spqr_adapters_pack.argtypes = C.c_int, [_vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp]
        lib.spqr_adapters_workspace_bytes.restype, lib.spqr_adapters_workspace_bytes.argtypes = _i64, [_vp, _i32]
        lib.spqr_token_logprobs_workspace_bytes.restype, lib.spqr_token_logprobs_workspace_bytes.argtypes = _i64, [_vp]
    return lib


def _run(name, index, stream, desc, *args):
    """One of the entries, on the handle's device: launches go to the current one, on its current stream where none is given."""
    if S._current_device() != index:
        import torch
        with torch.cuda.device(index):
            return _run(name, index, stream, desc, *args)
    rc = B._call(_entry[name], desc, *args, S._raw_stream(index) if stream is None else _address(stream, index))
    if rc != 0:
        raise SpQRError(int(rc), name)


def _address(stream, index):
    if stream.device_index != index:
        raise ValueError(f"a stream of cuda:{stream.device_index} for a handle on cuda:{index}")
    return stream.cuda_stream


def _on(stream, index):
    """A call's stream as the current one, for what the call makes (binding._on); of the handle's device."""
    _address(stream, index)
    return B._on(stream)


def _device(device):
    import torch
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError(f"a handle's arrays are in device memory, not on {device}")
    return torch.device("cuda", torch.cuda.current_device()) if device.index is None else device


def _stride(name, t, shape, index, dtype=None):
    """Elements between the rows of t, which has this shape, contiguous rows, and this type (None: any of the three)."""
    row, inner = t.stride() if t.dim() == 2 else (0, 0)
    if t.shape != shape or t.get_device() != index or (t.dtype not in S._dtypes if dtype is None else t.dtype != dtype):
        raise ValueError(f"{name}: {dtype or 'float32, float16 or bfloat16'} {list(shape)} on cuda:{index}, not {t.dtype} {list(t.shape)} on {t.device}")
    if inner != 1 and shape[1] > 1:
        raise ValueError(f"{name}: rows are contiguous, not with strides {list(t.stride())}")
    return row if shape[0] > 1 else shape[1]


class SpQRResidualNorm:
    """Norms around a block and what joins them, for rows of `width` elements:

        s = skip * x + scale * act(gate) * norm_y(y),   out = norm_x(s)

    norm_y, norm_x: None, "rms" or "layer", with weights and biases (device tensors [width] of one type, or None: 1 and 0;
    weight_offset is added to weights that are given).  act: None, "silu", "sigmoid" or "tanh", of the gate.  out_dtype: None for
    a call that only sums."""

    def __init__(self, width, *, norm_y=None, norm_x="rms", y_weight=None, y_bias=None, x_weight=None, x_bias=None, weight_offset=0.0, eps=1e-6,
                 skip=1.0, scale=1.0, act=None, out_dtype="float16", device="cuda"):
        import torch
        _lib()
        vectors = dict(y_weight=y_weight, y_bias=y_bias, x_weight=x_weight, x_bias=x_bias)
        given = {n: v for n, v in vectors.items() if v is not None}
        self.device = _device(next((v.device for v in given.values()), device))
        self._index, self.width = self.device.index, int(width)
        if isinstance(out_dtype, str):
            out_dtype = getattr(torch, out_dtype)
        if out_dtype is not None and out_dtype not in S._dtypes:
            raise ValueError(f"out_dtype: float32, float16, bfloat16 or None, not {out_dtype}")
        if norm_y not in _NORMS or norm_x not in _NORMS or act not in _ACTS:
            raise ValueError(f"norms are None, 'rms', 'layer', act is None, 'silu', 'sigmoid', 'tanh': not {norm_y!r}, {norm_x!r}, {act!r}")
        self.out_dtype = out_dtype
        d = self.desc = spqr_residual_norm_t()
        d.width, d.norm_y, d.norm_x, d.act = self.width, _NORMS[norm_y], _NORMS[norm_x], _ACTS[act]
        d.eps, d.weight_offset, d.skip, d.scale = float(eps), float(weight_offset), float(skip), float(scale)
        self._out_type = 0 if out_dtype is None else S._dtypes[out_dtype]
        self._one = None if out_dtype is None else torch.empty(1, dtype=out_dtype, device=self.device)
        dtype = next((v.dtype for v in given.values()), torch.float32)
        for n, v in given.items():
            if v.dtype != dtype or dtype not in S._dtypes or tuple(v.shape) != (self.width,) or not v.is_contiguous() or v.device != self.device:
                raise ValueError(f"{n}: a contiguous tensor [{self.width}] on {self.device}, all four of one type, not {v.dtype} {list(v.shape)} on {v.device}")
            setattr(d, n, v.data_ptr())
        d.weight_dtype = S._dtypes[dtype]
        self._vectors = vectors                  # alive as long as the descriptor


def spqr_residual_norm(norm: SpQRResidualNorm, x=None, y=None, gate=None, *, sum=None, out=None, stream=None):
    """(s, norm_x(s)) of rows x, y [rows, width] (one may be None); gate [width] or [rows, width], or None.  s, in x's type, is
    made where there are both x and y, or written to `sum` (which may be x); else None.  The norm, of the handle's out_dtype, is made or
    written to `out`; None with out_dtype None."""
    index, dtypes = norm._index, S._dtypes
    if stream is not None and ((sum is None and x is not None and y is not None) or (out is None and norm.out_dtype is not None)):
        with _on(stream, index):
            return spqr_residual_norm(norm, x, y, gate, sum=sum, out=out)
    rows = y if x is None else x
    if rows is None or rows.dim() != 2:
        raise ValueError("x, y: [rows, width], one of them at least")
    shape = rows.shape
    count, width = shape
    if width != norm.width:
        raise ValueError(f"rows of {norm.width} elements, not {list(shape)}")
    x_at = y_at = gate_at = sum_at = out_at = x_stride = y_stride = gate_stride = sum_stride = 0
    x_type = y_type = gate_type = 0
    if x is not None:
        x_stride, x_type, x_at = _stride("x", x, shape, index), dtypes[x.dtype], x.data_ptr()
    if y is not None:
        y_stride, y_type, y_at = _stride("y", y, shape, index), dtypes[y.dtype], y.data_ptr()
    if gate is not None:
        if y is None:
            raise ValueError("a gate without y")
        if gate.dim() == 1:
            _stride("gate", gate[None], (1, width), index)
        else:
            gate_stride = _stride("gate", gate, shape, index)
        gate_type, gate_at = dtypes[gate.dtype], gate.data_ptr()
    if sum is None:
        if x is not None and y is not None:
            sum = _empty_like(x) if x_stride == width else _empty(shape, dtype=x.dtype, device=x.device)
            sum_at, sum_stride = sum.data_ptr(), width
    else:
        sum_stride, x_type, sum_at = _stride("sum", sum, shape, index, None if x is None else x.dtype), dtypes[sum.dtype], sum.data_ptr()
    out_stride = width
    if norm.out_dtype is None:
        if out is not None:
            raise ValueError("out: this handle has out_dtype None")
    else:
        if out is None:
            out = norm._one.new_empty(shape)
        else:
            out_stride = _stride("out", out, shape, index, norm.out_dtype)
        out_at = out.data_ptr()
    d = norm.desc
    _norm_types.pack_into(d, 0, count, width, x_type, y_type, gate_type, norm._out_type)
    _norm_rows.pack_into(d, _norm_rows_at, x_at, y_at, gate_at, sum_at, out_at, x_stride, y_stride, sum_stride, out_stride, gate_stride)
    _run("spqr_residual_norm", index, stream, d)
    return sum, out


class SpQRAdapterPlan:
    """Which rows of a step go through which adapter: filled by spqr_adapter_plan, once a step, read by spqr_adapters.  rows: the
    step's; slots: places of the banks.  count [1], tile [max_tiles, 2] (slot, rows) and row [max_tiles, 64] are device tensors
    (int32) that stay where they are."""

    def __init__(self, rows, slots, device="cuda"):
        import torch
        tiles = _lib().spqr_adapter_tiles(int(rows), int(slots))
        if tiles < 0:
            raise SpQRError(tiles, "spqr_adapter_tiles")
        self.rows, self.slots, self.device = int(rows), int(slots), _device(device)
        self._index = self.device.index
        buffer = torch.full((64 + tiles * (SPQR_ADAPTER_TILE + 2),), -1, dtype=torch.int32, device=self.device)
        buffer[0] = 0
        self.count, self.row = buffer[:1], buffer[64:64 + 64 * tiles].view(tiles, SPQR_ADAPTER_TILE)
        self.tile = buffer[64 + 64 * tiles:].view(tiles, 2)
        d = self.desc = spqr_adapter_plan_t(rows=self.rows, slots=self.slots, max_tiles=tiles, count=self.count.data_ptr(), tile=self.tile.data_ptr(),
                                            row=self.row.data_ptr())
        self._at = C.addressof(d)
        _wait_for(self.device)


def spqr_adapter_plan(plan: SpQRAdapterPlan, adapter, q_start=None, stream=None) -> SpQRAdapterPlan:
    """The step's rows by adapter.  adapter: int32 [requests], the slot of each request (anything outside: none), with q_start int32
    [requests + 1] (SpQRStep.q_start); or [rows], without."""
    d, index = plan.desc, plan._index
    for name, a, n in (("adapter", adapter, plan.rows if q_start is None else adapter.numel()), ("q_start", q_start, adapter.numel() + 1)):
        if a is not None and (a.dtype != S._int32 or not a.is_contiguous() or a.dim() != 1 or a.numel() != n or a.get_device() != index):
            raise ValueError(f"{name}: a contiguous int32 tensor [{n}] on {plan.device}, not {a.dtype} {list(a.shape)} on {a.device}")
    d.requests, d.adapter, d.q_start = adapter.numel(), adapter.data_ptr(), None if q_start is None else q_start.data_ptr()
    _run("spqr_adapter_plan", index, stream, d)
    return plan


class SpQRAdapters:
    """Banks of low-rank adapters for projections that share their input, packed from A[p] [slots, max_rank, width] and B[p] [slots, m,
    max_rank], all float16 or all bfloat16 (max_rank and m may differ from projection to projection; A and B are not needed
    afterwards).  rank: int32 [slots], one for all projections, a list of one each, or None (max_rank).  scale: the same, float32
    [slots], read by each call; None: 1.  rows: of the largest step, which the scratch is made for; workspace: a device tensor to use instead
    (banks that are called one after the other may share it)."""

    def __init__(self, A, B, rank=None, scale=None, *, rows, workspace=None):
        import torch
        lib = _lib()
        A, B = list(A), list(B)
        k = len(A)
        if k < 1 or k > SPQR_MAX_FUSED or len(B) != k:
            raise ValueError(f"as many A as B, 1 to {SPQR_MAX_FUSED}")
        d = self.desc = spqr_adapters_t()
        self.device, self.dtype, self.rows = A[0].device, A[0].dtype, int(rows)
        if self.device.type != "cuda" or self.dtype not in (torch.float16, torch.bfloat16) or any(t.dim() != 3 for t in A + B):
            raise ValueError("A, B: float16 or bfloat16 device tensors [slots, max_rank, width], [slots, m, max_rank]")
        self._index = self.device.index
        self.slots, self.width = A[0].shape[0], A[0].shape[2]
        self.m, self.max_rank = [b.shape[1] for b in B], [a.shape[1] for a in A]
        scale = [scale] * k if scale is None or hasattr(scale, "dtype") else list(scale)
        if len(scale) != k:
            raise ValueError(f"scale: one, or {k}")
        for t in scale:
            if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (self.slots,) or not t.is_contiguous() or t.device != self.device):
                raise ValueError(f"scale: a contiguous float32 tensor [{self.slots}] on {self.device}")
        self.scale = scale
        d.count, d.width, d.slots, d.dtype = k, self.width, self.slots, S._dtypes[self.dtype]
        for p in range(k):
            d.max_rank[p], d.m[p], d.scale[p] = self.max_rank[p], self.m[p], None if scale[p] is None else scale[p].data_ptr()
        self.banks = []
        for p in range(k):
            need = int(lib.spqr_adapters_bank_bytes(C.byref(d), p))
            if need < 0:
                raise SpQRError(need, "spqr_adapters_bank_bytes")
            self.banks.append(torch.empty(need, dtype=torch.uint8, device=self.device))
            d.bank[p] = self.banks[p].data_ptr()
        need = int(lib.spqr_adapters_workspace_bytes(C.byref(d), self.rows))
        if need < 0:
            raise SpQRError(need, "spqr_adapters_workspace_bytes")
        if workspace is None:
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        elif workspace.device != self.device or not workspace.is_contiguous():
            raise ValueError(f"workspace: a contiguous tensor on {self.device}")
        self.workspace = workspace
        d.workspace, d.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        self.load(0, A, B, rank)
        _wait_for(self.device)

    def load(self, first, A, B, rank=None, stream=None):
        """Other adapters into the slots from `first` on: A, B and rank as above, of as many slots as are to be filled (not needed after the call,
        on another stream neither)."""
        import torch
        k, A, B = len(self.m), list(A), list(B)
        rank = [rank] * k if rank is None or hasattr(rank, "dtype") else list(rank)
        if stream is not None:
            with _on(stream, self._index):
                self.load(first, A, B, rank)
            for t in A + B + rank:
                if t is not None:
                    t.record_stream(stream)
            return
        if len(A) != k or len(B) != k or len(rank) != k:
            raise ValueError(f"A, B: {k} tensors; rank: one, or {k}")
        slots = A[0].shape[0]
        if first < 0 or first + slots > self.slots:
            raise ValueError(f"slots {first} .. {first + slots - 1} of {self.slots}")
        for p in range(k):
            for t, name, shape in ((A[p], "A", (slots, self.max_rank[p], self.width)), (B[p], "B", (slots, self.m[p], self.max_rank[p]))):
                if t.dtype != self.dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != self.device:
                    raise ValueError(f"{name}[{p}]: a contiguous {self.dtype} tensor {list(shape)} on {self.device}, not {t.dtype} {list(t.shape)} on {t.device}")
            t = rank[p]
            if t is not None and (t.dtype != torch.int32 or tuple(t.shape) != (slots,) or not t.is_contiguous() or t.device != self.device):
                raise ValueError(f"rank: a contiguous int32 tensor [{slots}] on {self.device}")
        lib = _lib()
        with torch.cuda.device(self._index):
            to = S._raw_stream(self._index)
            for p in range(k):
                rc = lib.spqr_adapters_pack(C.byref(self.desc), p, first, slots, A[p].data_ptr(), B[p].data_ptr(), None if rank[p] is None else rank[p].data_ptr(), to)
                if rc != 0:
                    raise SpQRError(int(rc), "spqr_adapters_pack")


def spqr_adapters(bank: SpQRAdapters, plan: SpQRAdapterPlan, x, ys=None, outs=None, stream=None):
    """outs[p] = ys[p] + scale B[p] (A[p] x), row by row by the plan's adapters: x [rows, width] of the banks' type, ys and outs
    [rows, m[p]] of one type.  ys None: zeros (outs are float32 unless given).  outs None: new tensors; outs may be ys.  Rows that the
    plan has in no tile are left as they are."""
    d, index, dtypes = bank.desc, bank._index, S._dtypes
    if stream is not None and outs is None:
        with _on(stream, index):
            return spqr_adapters(bank, plan, x, ys)
    rows, k, ms = plan.rows, len(bank.m), bank.m
    if plan._index != index:
        raise ValueError(f"a plan on {plan.device}, banks on {bank.device}")
    d.x_stride, d.x = _stride("x", x, (rows, bank.width), index, bank.dtype), x.data_ptr()
    if (ys is not None and len(ys) != k) or (outs is not None and len(outs) != k):
        raise ValueError(f"ys, outs: {k} tensors")
    fields = [0] * (4 * SPQR_MAX_FUSED)
    first = (outs or ys)
    dtype = _float32 if first is None else first[0].dtype
    if dtype not in dtypes:
        raise ValueError(f"ys, outs: float32, float16 or bfloat16, not {dtype}")
    if ys is not None:
        for p in range(k):
            fields[2 * SPQR_MAX_FUSED + p] = _stride("ys", ys[p], (rows, ms[p]), index, dtype)
            fields[p] = ys[p].data_ptr()
    if outs is None:
        outs = [_empty((rows, m), dtype=dtype, device=x.device) if ys is None or fields[2 * SPQR_MAX_FUSED + p] != m else _empty_like(ys[p])
                for p, m in enumerate(ms)]
        fields[3 * SPQR_MAX_FUSED:3 * SPQR_MAX_FUSED + k] = ms
    else:
        for p in range(k):
            fields[3 * SPQR_MAX_FUSED + p] = _stride("outs", outs[p], (rows, ms[p]), index, dtype)
    for p in range(k):
        fields[SPQR_MAX_FUSED + p] = outs[p].data_ptr()
    _bank_rows.pack_into(d, _bank_rows_at, *fields)
    d.y_dtype = dtypes[dtype]
    _run("spqr_adapters", index, stream, d, plan._at)
    return outs


class SpQRScores:
    """Log probabilities of rows of logits, and room for them: logprob [rows, given], entropy [rows], top_token (int32) and
    top_logprob [rows, top], which each call of spqr_token_logprobs overwrites.  rows: the most of a call."""

    def __init__(self, rows, vocab, *, given=1, top=0, device="cuda"):
        import torch
        lib = _lib()
        self.rows, self.vocab, self.given, self.top, self.device = int(rows), int(vocab), int(given), int(top), _device(device)
        self._index = self.device.index
        d = self.desc = spqr_token_logprobs_t(rows=self.rows, vocab=self.vocab, given=self.given, top=self.top)
        need = int(lib.spqr_token_logprobs_workspace_bytes(C.byref(d)))
        if need < 0:
            raise SpQRError(need, "spqr_token_logprobs_workspace_bytes")
        self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        d.workspace, d.workspace_bytes = self.workspace.data_ptr(), self.workspace.numel()
        empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=self.device)  # noqa: E731
        self.logprob, self.entropy = empty(self.rows, self.given), empty(self.rows)
        self.top_token, self.top_logprob = empty(self.rows, self.top, dtype=torch.int32), empty(self.rows, self.top)
        for n in ("logprob", "entropy", "top_token", "top_logprob"):
            setattr(d, n, getattr(self, n).data_ptr())
        _wait_for(self.device)


def spqr_token_logprobs(scores: SpQRScores, logits, tokens=None, scale: float = 1.0, stream=None) -> SpQRScores:
    """Fills `scores` for logits [rows, vocab] (float32, float16, bfloat16): log softmax(scale * logits) of tokens int32 [rows, given]
    ([rows] where given is 1), entropies, the most probable tokens.  Fewer rows than the handle's: the first ones are filled."""
    d, index = scores.desc, scores._index
    if logits.dim() != 2 or logits.shape[0] > scores.rows:
        raise ValueError(f"logits: up to {scores.rows} rows of {scores.vocab}, not {list(logits.shape)}")
    rows = logits.shape[0]
    d.stride, d.dtype, d.logits, d.rows = _stride("logits", logits, (rows, scores.vocab), index), S._dtypes[logits.dtype], logits.data_ptr(), rows
    if scores.given:
        if (tokens is None or tokens.dtype != S._int32 or tokens.numel() != rows * scores.given or not tokens.is_contiguous() or tokens.get_device() != index
                or (scores.given > 1 and tokens.dim() == 2 and tokens.shape[0] != rows)):
            raise ValueError(f"tokens: a contiguous int32 tensor [{rows}, {scores.given}] on {scores.device}")
        d.tokens = tokens.data_ptr()
    elif tokens is not None:
        raise ValueError("tokens: this handle has given = 0")
    d.scale = scale
    _run("spqr_token_logprobs", index, stream, d)
    return scores
