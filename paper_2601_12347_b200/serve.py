"""Operators that answer requests from the cached rows: include/ripple.h, "Requests".

A request names vertices; what it wants is a learned head run on their rows.  The head is a stack of residual blocks
(norm, projection, norm, gate, scale, sum), its projections shared by all tenants, with a low-rank adapter of the
request's tenant beside each:

    norm_rows      s = residual[ids] + scale * act(gate) * post(y);   n = pre(s)
    project_rows   y = act(x[ids] W + bias + scale_a (x[ids] A_a) B_a),  a = the row's slot of the bank
    RequestHead    a stack of such blocks over the rows of one layer; `Ripple.answer` runs it

Everything runs on the current CUDA stream of the tensors' device (not necessarily the current device) and returns once
it is launched; calls can be captured into CUDA graphs.  Device-side waits are bounded; a call whose wait gave up has returned long
before, and its results are not to be used: `check_requests`, where a program waits for its results anyway, tells of it.  Outputs and scratch come from PyTorch's allocator, so every call
and every captured graph has its own.  Operators (Norm, Projection, AdapterBank, RequestHead) may be dropped while calls that read them
are in flight, on whatever stream; tensors of the caller follow PyTorch's rule (`Tensor.record_stream`), and a captured graph reads
both as long as it is replayed.  Rows whose id lies outside the table (a negative id marks padding) are not
written: they keep what `out` holds, and without `out` what the memory of the result held (a RequestHead's hold what it makes of zeros).  Rows are fp32, bf16 or fp16; sums and statistics are fp32.  The library infers: inputs that
require gradients are refused while gradients are recorded, and inputs that carry tangents always.
"""
from __future__ import annotations

import ctypes
import struct
from dataclasses import dataclass
from typing import List, Optional, Sequence, Tuple, Union

import numpy as np
import torch
from torch.autograd import forward_ad

from . import ripple as _ripple
from .ripple import ACT_IDENTITY, ACT_RELU, OK, RippleError

TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2
GATE_IDENTITY, GATE_SIGMOID, GATE_SILU, GATE_TANH = 0, 1, 2, 3
MAX_RANK, MAX_SLOTS = 64, 4096

_TYPES = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}
# ripple_norm_rows_args, ripple_project_rows_args
_NORM_ARGS = struct.Struct("=q4i QqQqQqqQQQqQq ifQQ ifQQ f3i Q")
_PROJECT_ARGS = struct.Struct("=q8i QqqQQQQQQq Qq Q")


def _check(status: int) -> None:
    if status != OK:
        raise RippleError(status, _ripple.load_library().ripple_last_error(None).decode())


def _type_of(dtype, name: str) -> int:
    t = _TYPES.get(dtype)
    if t is None:
        raise TypeError(f"{name}: float32, bfloat16 or float16 expected, got {dtype}")
    return t


# A call of a few rows takes a few microseconds on the device; what is checked here before it is therefore checked with as few
# calls into PyTorch as it can be, and explained only where it fails.
def _refuse(t, name: str, index: int):
    """Why a tensor is not one that the device `index` (-1: any) can read."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: a CUDA tensor expected, got {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor expected, it is on {t.device}")
    if index >= 0 and t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, the other tensors on cuda:{index}")
    raise ValueError(f"{name} requires gradients, which these operators do not form: call them under torch.no_grad()")


def _refuse_tangents(**tensors) -> None:
    """Within a level of forward-mode differentiation: no input may carry a tangent, which would be dropped."""
    for name, t in tensors.items():
        if isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError(f"{name} carries a tangent, which these operators do not form")


def _device_of(t, name: str) -> int:
    index = t.get_device() if isinstance(t, torch.Tensor) else -1
    if index < 0 or not t.is_cuda:
        _refuse(t, name, -1)
    return index


def _matrix(t, name: str, width: Optional[int], dtype, index: int) -> Tuple[int, int, int]:
    """Address, leading dimension and rows of a matrix whose columns lie side by side."""
    if not isinstance(t, torch.Tensor) or t.get_device() != index or (t.requires_grad and torch.is_grad_enabled()):
        _refuse(t, name, index)
    shape = t.shape
    if len(shape) != 2 or (width is not None and shape[1] != width):
        raise ValueError(f"{name}: [rows, {'columns' if width is None else width}] expected, got {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: {dtype} expected, got {t.dtype}")
    rows, cols = shape
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        raise ValueError(f"{name}: the columns of a row must lie side by side, the stride is {inner}")
    return t.data_ptr(), (ld if rows > 1 else max(cols, 1)), rows


def _vector(t, name: str, size: int, dtype, index: int) -> int:
    if not isinstance(t, torch.Tensor) or t.get_device() != index or (t.requires_grad and torch.is_grad_enabled()):
        _refuse(t, name, index)
    if t.dtype != dtype:
        raise TypeError(f"{name}: {dtype} expected, got {t.dtype}")
    if t.shape != (size,) or (size > 1 and t.stride(0) != 1):
        raise ValueError(f"{name}: [{size}], contiguous, expected, got {tuple(t.shape)} of stride {t.stride()}")
    return t.data_ptr()


def _to_device(a, dtype, device, name: str, copy: bool = False):
    """A weight given as an array or a tensor, contiguous on the device; with `copy` never the caller's memory."""
    if isinstance(a, torch.Tensor):
        if device is None and a.is_cuda:
            device = a.device
        a = a.detach()
    else:
        a = torch.from_numpy(np.ascontiguousarray(a))
    if not a.is_floating_point():
        raise TypeError(f"{name}: floating-point values expected, got {a.dtype}")
    device = torch.device("cuda") if device is None else torch.device(device)
    if device.type != "cuda":
        raise ValueError(f"{name}: a CUDA device expected, got {device}")
    if device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    return a.to(device=device, dtype=dtype or a.dtype, copy=copy).contiguous()


def _stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


# (the same number without an object around it, where PyTorch has it)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream)


class _Buffers:
    """Device memory that an operator keeps.  It belongs to the stream that it was allocated on; PyTorch's allocator is told of every
    other that a call reads it on, so that an operator may be dropped while such calls are in flight.  (Once per stream: what counts is
    where the stream stands when the memory is given back.)"""

    def _keep(self, index: Optional[int], *tensors):
        self._tensors = tensors
        self._streams = set() if index is None else {_stream(index)}

    # (A deep copy or a pickled one would hold the addresses of this one's memory and not keep it.)
    def __reduce_ex__(self, protocol):
        raise TypeError(f"a {type(self).__name__} holds device memory and cannot be copied or pickled: make another from its weights")

    def __copy__(self):
        other = object.__new__(type(self))
        other.__dict__.update(self.__dict__)
        return other

    def _read_on(self, stream: int):
        if stream in self._streams:
            return
        for t in self._tensors:
            with torch.cuda.device(t.device):
                if torch.cuda.is_current_stream_capturing():
                    return                     # (nothing is in flight; who replays the graph keeps the operator)
                t.record_stream(torch.cuda.current_stream())
        self._streams.add(stream)


class Norm(_Buffers):
    """Layer or root-mean-square norm with its vectors (arrays or tensors; an fp32 copy is kept on the device)."""

    def __init__(self, kind: int, weight=None, bias=None, eps: float = 1e-5, device=None):
        if kind not in (NORM_LAYER, NORM_RMS):
            raise ValueError(f"kind: NORM_LAYER or NORM_RMS expected, got {kind}")
        if not eps >= 0:
            raise ValueError(f"eps: {eps}")
        self.kind, self.eps = int(kind), float(eps)
        self.weight = None if weight is None else _to_device(weight, torch.float32, device, "weight", copy=True)
        self.bias = None if bias is None else _to_device(bias, torch.float32, device, "bias", copy=True)
        self.width = self.index = None         # any, without vectors
        for t in (self.weight, self.bias):
            if t is not None:
                if t.dim() != 1 or self.width not in (None, t.shape[0]) or self.index not in (None, t.get_device()):
                    raise ValueError("norm vectors: one dimension, one size and one device expected")
                self.width, self.index = t.shape[0], t.get_device()
                torch.cuda.current_stream(t.device).synchronize()    # usable on every stream from here on
        self._keep(self.index, *(t for t in (self.weight, self.bias) if t is not None))
        self._args = (self.kind, self.eps, 0 if self.weight is None else self.weight.data_ptr(), 0 if self.bias is None else self.bias.data_ptr())

    def _packed(self, width: int, index: int, stream: int, name: str):
        if self.width is not None and (self.width != width or self.index != index):
            raise ValueError(f"{name}: vectors of {width} entries on cuda:{index} expected, got {self.width} on cuda:{self.index}")
        self._read_on(stream)
        return self._args


_NO_NORM = (NORM_NONE, 0.0, 0, 0)


def norm_rows(y=None, *, post: Optional[Norm] = None, gate=None, gate_act: int = GATE_IDENTITY, scale=1.0,
              residual=None, ids=None, pre: Optional[Norm] = None, normed_dtype=None, out=None, normed_out=None, clear_padding: bool = False):
    """(s, n):  s = residual[ids] + scale * act(gate) * post(y),  n = pre(s);  n is None without `pre`.

    y [rows, D]: a block's output; without it s = residual[ids], which is returned only if `out` or no `pre` is given.
    gate [rows, D] or [rows, 1], of y's type; scale: a number, or an fp32 vector [D].
    residual [any, D]: y's type or fp32; row ids[i] (int32) of it, or row i, goes to row i; without it s = scale * ...
    s has residual's type, n y's (without y: normed_dtype, or residual's).  out / normed_out: where to write s / n; they may be y,
    or residual if there are no ids, but overlap no input otherwise.  clear_padding: the rows of ids outside the residual become zeros."""
    if y is None and residual is None:
        raise ValueError("neither y nor residual")
    if getattr(forward_ad, "_current_level", 0) >= 0:
        _refuse_tangents(y=y, gate=gate, scale=scale, residual=residual, out=out, normed_out=normed_out)
    first, name = (y, "y") if y is not None else (residual, "residual")
    index = _device_of(first, name)
    ptr, ld, rows = _matrix(first, name, None, None, index)
    width = first.shape[1]
    ids_ptr = gate_ptr = gate_ld = res_ptr = res_ld = res_rows = y_ptr = y_ld = vec_ptr = 0
    gate_width = 1
    if y is not None:
        y_ptr, y_ld, dtype = ptr, ld, y.dtype
        if normed_dtype is not None and normed_dtype != dtype:
            raise TypeError(f"normed_dtype: y's type, {dtype}, expected, got {normed_dtype}")
        if residual is not None:
            res_ptr, res_ld, res_rows = _matrix(residual, "residual", width, None, index)
            stream_dtype = residual.dtype
        else:
            stream_dtype = dtype
    else:
        if gate is not None or post is not None:
            raise ValueError("gate or post without y")
        res_ptr, res_ld, res_rows, stream_dtype = ptr, ld, rows, residual.dtype
        dtype = normed_dtype or stream_dtype
        if ids is not None:
            if getattr(ids, "dim", lambda: 0)() != 1:
                raise ValueError("ids: one dimension expected")
            rows = ids.shape[0]
    t, ts = _type_of(dtype, "y" if y is not None else "normed_dtype"), _type_of(stream_dtype, "residual")
    if ts != t and ts != TYPE_F32:
        raise TypeError(f"residual: {dtype} or float32 expected, got {stream_dtype}")
    if ids is not None:
        if residual is None:
            raise ValueError("ids without residual")
        ids_ptr = _vector(ids, "ids", rows, torch.int32, index)
    elif residual is not None and res_rows != rows:
        raise ValueError(f"residual: {rows} rows expected, got {res_rows}")
    if gate is not None:
        gate_ptr, gate_ld, gr = _matrix(gate, "gate", None, dtype, index)
        gate_width = gate.shape[1]
        if gate_width not in (1, width) or gr != rows:
            raise ValueError(f"gate: [{rows}, {width}] or [{rows}, 1] expected, got {tuple(gate.shape)}")
    number = 1.0
    if isinstance(scale, torch.Tensor):
        vec_ptr = _vector(scale, "scale", width, torch.float32, index)
    else:
        number = float(scale)
    out_ptr = out_ld = n_ptr = n_ld = 0
    if out is not None:
        out_ptr, out_ld, got = _matrix(out, "out", width, stream_dtype, index)
        if got != rows:
            raise ValueError(f"out: {rows} rows expected, got {got}")
    elif y is not None or pre is None:
        out = torch.empty((rows, width), dtype=stream_dtype, device=first.device)
        out_ptr, out_ld = out.data_ptr(), width
    if pre is not None:
        if normed_out is None:
            normed_out = torch.empty((rows, width), dtype=dtype, device=first.device)
            n_ptr, n_ld = normed_out.data_ptr(), width
        else:
            n_ptr, n_ld, got = _matrix(normed_out, "normed_out", width, dtype, index)
            if got != rows:
                raise ValueError(f"normed_out: {rows} rows expected, got {got}")
    elif normed_out is not None:
        raise ValueError("normed_out without pre")
    stream = _stream(index)
    post_args = _NO_NORM if post is None else post._packed(width, index, stream, "post")
    pre_args = _NO_NORM if pre is None else pre._packed(width, index, stream, "pre")
    if rows == 0 or (ids is not None and res_rows == 0):       # (without rows every id lies outside)
        for t in (out, normed_out):
            if clear_padding and t is not None:
                t.zero_()
        return out, normed_out
    _check(_ripple.load_library().ripple_norm_rows(_NORM_ARGS.pack(
        rows, width, t, ts, int(gate_act), y_ptr, y_ld, gate_ptr, gate_ld, res_ptr, res_ld, res_rows, ids_ptr, vec_ptr,
        out_ptr, out_ld, n_ptr, n_ld, *post_args, *pre_args, number, gate_width, index, bool(clear_padding), stream)))
    return out, normed_out


class Projection(_Buffers):
    """y = act(x W + bias), W [K, N] input-major like the layers' matrices, laid out once for the tensor cores.

    W, bias: arrays or tensors; `dtype` (default: W's) is the type of x, W and the adapters.  Copies are kept, of the bias in fp32."""

    def __init__(self, W, bias=None, act: int = ACT_IDENTITY, dtype=None, device=None):
        W = _to_device(W, dtype, device, "W")
        if W.dim() != 2:
            raise ValueError(f"W: [K, N] expected, got {tuple(W.shape)}")
        self.lib = _ripple.load_library()
        self.dtype, self.device, self.index = W.dtype, W.device, W.get_device()
        self.type = _type_of(W.dtype, "W")
        self.K, self.N = W.shape
        if act not in (ACT_IDENTITY, ACT_RELU):
            raise ValueError(f"act: ACT_IDENTITY or ACT_RELU expected, got {act}")
        self.act = int(act)
        size = self.lib.ripple_project_layout_bytes(self.type, self.K, self.N)
        if size < 0:
            raise ValueError(f"W: {self.K} x {self.N} is out of range")
        self.bias = None if bias is None else _to_device(bias, torch.float32, self.device, "bias", copy=True)
        if self.bias is not None and tuple(self.bias.shape) != (self.N,):
            raise ValueError(f"bias: [{self.N}] expected, got {tuple(self.bias.shape)}")
        self.layout = torch.empty(size, dtype=torch.uint8, device=self.device)
        _check(self.lib.ripple_project_layout(self.type, self.K, self.N, W.data_ptr(), self.N, self.layout.data_ptr(),
                                              self.index, _stream(self.index)))
        torch.cuda.current_stream(self.device).synchronize()     # usable on every stream from here on
        self._keep(self.index, *(t for t in (self.layout, self.bias) if t is not None))
        self._tail = (self.layout.data_ptr(), 0 if self.bias is None else self.bias.data_ptr())


class AdapterBank(_Buffers):
    """Low-rank adapters of one projection, by slot."""

    def __init__(self, projection: Projection, slots: int, max_rank: int):
        p = projection
        self.projection, self.slots, self.max_rank = p, int(slots), int(max_rank)
        if not 1 <= self.slots <= MAX_SLOTS or not 1 <= self.max_rank <= MAX_RANK:
            raise ValueError(f"1 to {MAX_SLOTS} slots of rank 1 to {MAX_RANK} expected, got {slots} of {max_rank}")
        self.buffer = torch.empty(p.lib.ripple_adapter_bytes(p.type, p.K, p.N, self.slots, self.max_rank), dtype=torch.uint8, device=p.device)
        self._keep(p.index, self.buffer)
        self._scratch = (-1, 0)          # rows of the last call, and the scratch that it takes
        self._set(0, self.slots, 0, None, None, None)

    def _set(self, first, count, rank, A, B, scale):
        p = self.projection
        _check(p.lib.ripple_adapter_set(self.buffer.data_ptr(), p.type, p.K, p.N, self.slots, self.max_rank, first, count, rank,
                                        None if A is None else A.data_ptr(), None if B is None else B.data_ptr(), scale,
                                        p.index, _stream(p.index)))

    def set(self, slot: int, A, B, scale: Union[float, Sequence[float]] = 1.0) -> None:
        """A [K, r], B [r, N] into `slot`; or A [m, K, r], B [m, r, N], scale: m numbers (or one for all) into `slot` and those
        behind it.  Returns once they are in place; refuses entries that are not finite (the slots are then empty).  No call that reads the bank may be in
        flight on another stream."""
        p = self.projection
        A, B = _to_device(A, p.dtype, p.device, "A"), _to_device(B, p.dtype, p.device, "B")
        if A.dim() == 2:
            A = A[None]
        if B.dim() == 2:
            B = B[None]
        if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[2] != B.shape[1] or A.shape[1] != p.K or B.shape[2] != p.N:
            raise ValueError(f"A [m, {p.K}, r] and B [m, r, {p.N}] expected, got {tuple(A.shape)} and {tuple(B.shape)}")
        m, _, rank = A.shape
        if not 1 <= rank <= self.max_rank:
            raise ValueError(f"rank 1 to {self.max_rank} expected, got {rank}")
        if not 0 <= slot <= self.slots - m:
            raise ValueError(f"slots {slot} to {slot + m - 1} of {self.slots}")
        scales = [float(scale)] * m if not hasattr(scale, "__len__") else [float(x) for x in scale]
        if len(scales) != m:
            raise ValueError(f"scale: {m} numbers expected, got {len(scales)}")
        self._set(int(slot), m, rank, A, B, (ctypes.c_float * max(m, 1))(*scales))

    def clear(self, slot: int) -> None:
        if not 0 <= slot < self.slots:
            raise ValueError(f"slot {slot} of {self.slots}")
        self._set(int(slot), 1, 0, None, None, None)


def project_rows(x, projection: Projection, bank: Optional[AdapterBank] = None, slots=None, ids=None, out=None, out_dtype=None):
    """act(x[ids] W + bias + scale_a (x[ids] A_a) B_a) for every row, a = slots[i] (int32; a slot that is negative, out of
    range or empty: no adapter).  x [any, K] of the projection's type, ids int32 or None; the result has that type, or fp32 if
    out_dtype (or out) says so.  `out` shares no memory with an input.  Any order of slots is right; above a few thousand rows, rows of
    one slot side by side are fastest."""
    p = projection
    index = p.index
    if getattr(forward_ad, "_current_level", 0) >= 0:
        _refuse_tangents(x=x, out=out)
    x_ptr, x_ld, x_rows = _matrix(x, "x", p.K, p.dtype, index)
    rows, ids_ptr, bank_ptr, slots_ptr, n_slots, max_rank = x_rows, 0, 0, 0, 0, 0
    if ids is not None:
        if getattr(ids, "dim", lambda: 0)() != 1:
            raise ValueError("ids: one dimension expected")
        rows = ids.shape[0]
        ids_ptr = _vector(ids, "ids", rows, torch.int32, index)
    if (bank is None) != (slots is None):
        raise ValueError("bank and slots go together")
    if bank is not None:
        if bank.projection is not p:
            raise ValueError("the bank belongs to another projection")
        bank_ptr, n_slots, max_rank = bank.buffer.data_ptr(), bank.slots, bank.max_rank
        slots_ptr = _vector(slots, "slots", rows, torch.int32, index)
    if out is None:
        out = torch.empty((rows, p.N), dtype=out_dtype or p.dtype, device=p.device)
        y_ptr, y_ld = out.data_ptr(), p.N
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out: {out_dtype} expected, got {out.dtype}")
        y_ptr, y_ld, got = _matrix(out, "out", p.N, None, index)
        if got != rows:
            raise ValueError(f"out: {rows} rows expected, got {got}")
    out_type = p.type if out.dtype == p.dtype else _type_of(out.dtype, "out")
    if out_type not in (p.type, TYPE_F32):
        raise TypeError(f"out: {p.dtype} or float32 expected, got {out.dtype}")
    if rows == 0 or x_rows == 0:
        return out
    stream = _stream(index)
    p._read_on(stream)
    if bank is not None:
        bank._read_on(stream)
    head = (rows, p.type, out_type, p.K, p.N, p.act, n_slots, max_rank, index, x_ptr, x_ld, x_rows, ids_ptr, *p._tail, bank_ptr,
            slots_ptr, y_ptr, y_ld)
    need = work_ptr = 0
    if bank_ptr:
        known, need = bank._scratch
        if known != rows:
            need = p.lib.ripple_project_workspace_bytes(_PROJECT_ARGS.pack(*head, 0, 0, 0))
            bank._scratch = (rows, need)
        if need > 0:
            work = torch.empty(need, dtype=torch.uint8, device=p.device)     # of this call: the allocator keeps it until the stream has passed it
            work_ptr = work.data_ptr()
    _check(p.lib.ripple_project_rows(_PROJECT_ARGS.pack(*head, work_ptr, need, stream)))
    return out


def check_requests(device=None) -> None:
    """Waits for the device; raises RippleError (ERR_TIMEOUT) if a bounded device-side wait of a call (project_rows, a RequestHead,
    Ripple.answer; of train.py the losses) gave up since the last check: the results since then are not to be used.  No other call tells."""
    index = torch.cuda.current_device() if device is None else torch.device(device).index
    _check(_ripple.load_library().ripple_request_status(-1 if index is None else index))


@dataclass
class Block:
    """s + scale * post(down(up(pre(s)))): a residual block of a RequestHead.  `up` and `down` with their banks (or None)."""
    pre: Norm
    up: Projection
    down: Projection
    up_bank: Optional[AdapterBank] = None
    down_bank: Optional[AdapterBank] = None
    post: Optional[Norm] = None
    scale: Union[float, "torch.Tensor"] = 1.0


class RequestHead(_Buffers):
    """A head that requests run on the cached rows of their vertices: residual blocks, a last norm, the logits' projection.

    The residual stream starts from the fp32 rows of the cache and stays fp32; the blocks run in the projections' type."""

    def __init__(self, blocks: Sequence[Block], norm: Norm, logits: Projection, logits_bank: Optional[AdapterBank] = None):
        self.blocks: List[Block] = list(blocks)
        self.norm, self.logits, self.logits_bank = norm, logits, logits_bank
        for i, b in enumerate(self.blocks):
            if b.up.N != b.down.K or b.down.N != b.up.K or b.up.dtype != b.down.dtype or b.up.dtype != logits.dtype or b.up.K != logits.K:
                raise ValueError(f"block {i}: the widths or types of its projections do not fit")
        self._keep(None, *(b.scale for b in self.blocks if isinstance(b.scale, torch.Tensor)))

    def __call__(self, table, ids, slots=None, out_dtype=torch.float32):
        """Logits [len(ids), N] of the rows `ids` (int32) of `table`, each with the adapters of its slot (without slots: of the
        shared projections alone).  A row whose id lies outside the table enters every norm that gathers as zeros."""
        def project(x, p, bank, **kw):
            return project_rows(x, p, bank, slots, **kw) if bank is not None and slots is not None else project_rows(x, p, **kw)

        self._read_on(_stream(self.logits.index))
        first = self.blocks[0].pre if self.blocks else self.norm
        _, n = norm_rows(residual=table, ids=ids, pre=first, normed_dtype=self.logits.dtype, clear_padding=True)
        s, at = table, ids
        for i, b in enumerate(self.blocks):
            y = project(project(n, b.up, b.up_bank), b.down, b.down_bank)
            following = self.blocks[i + 1].pre if i + 1 < len(self.blocks) else self.norm
            s, n = norm_rows(y, post=b.post, scale=b.scale, residual=s, ids=at, pre=following, clear_padding=True)
            at = None
        return project(n, self.logits, self.logits_bank, out_dtype=out_dtype)
