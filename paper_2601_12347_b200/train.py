"""Operators that train a head on the cached rows: include/ripple.h, "Training".

What requests run (serve.py) has weights; these are fitted here, minibatch by minibatch, to labels of some vertices:

    lookup_rows        y_i = scale * table[ids_i]:  learned rows beside the cached ones
    lookup_rows_grad   dtable[r] = scale * sum of dy_i over the i with ids_i = r
    norm_rows_grad     dx, dweight, dbias of n = norm(x[ids]) (serve.norm_rows)
    loss_rows          softmax cross entropy of x W + bias over many classes, without the logits in memory
    loss_rows_grad     dx, dW, dbias of it
    ClassHead          a norm and a linear layer over the classes of vertices, with learned rows beside the cached ones: a step is a
                       run of these calls; `Ripple.train_step` takes it on the rows of a context

Gradients are calls of their own; nothing is recorded, and inputs that require gradients are refused while PyTorch records them (call
under torch.no_grad() or with detached tensors).  As with requests everything runs on the current CUDA stream of the tensors' device (not
necessarily the current device) and returns once it is launched; calls can be captured into CUDA graphs; outputs and scratch come from PyTorch's
allocator, so every call and every captured graph has its own.  Sums are fp32 and formed in a fixed order: the same call gives the same
bits.  Rows are fp32, bf16 or fp16.  Padding (ids or labels outside their range, -1 by custom) gives rows of zeros and adds nothing to
any gradient, whatever its rows hold.  Device-side waits of the losses are bounded; `serve.check_requests` tells whether one gave up.
"""
from __future__ import annotations

import struct
from functools import lru_cache
from typing import Dict

import torch
from torch.autograd import forward_ad

from . import ripple as _ripple
from .serve import (NORM_LAYER, NORM_RMS, TYPE_F32, Norm, Projection, RequestHead, _check, _device_of, _matrix, _refuse_tangents, _stream,
                    _type_of, _vector, norm_rows)

# ripple_lookup_rows_args, ripple_lookup_rows_grad_args, ripple_norm_rows_grad_args
_LOOKUP_ARGS = struct.Struct("=q4i QqqQ Qq fi Q")
_LOOKUP_GRAD_ARGS = struct.Struct("=q4i QqQ Qqq fi Qq Q")
_NORM_GRAD_ARGS = struct.Struct("=q4i Qq QqqQ Qq Qq QQ ifQQ Qq Q")
# ripple_live_rows_args, ripple_loss_rows_args, ripple_loss_rows_grad_args
_LIVE_ARGS = struct.Struct("=q2i Qq QQQQ Q")
_LOSS_ARGS = struct.Struct("=q4i QqQq QQQQ Qq Q")
_LOSS_GRAD_ARGS = struct.Struct("=q4i QqQq QQQQ QqQqQ fi Qq Q")


def _ids(ids, index: int):
    if getattr(ids, "dim", lambda: 0)() != 1:
        raise ValueError("ids: one dimension expected")
    rows = ids.shape[0]
    return _vector(ids, "ids", rows, torch.int32, index), rows


def _workspace(need: int, like):
    """Scratch of one call, from the allocator: it keeps the memory until the stream has passed the call."""
    return torch.empty(need, dtype=torch.uint8, device=like.device) if need > 0 else None


# Bytes of scratch, by sizes (and how matrices are aligned): asked of the library once for each.
@lru_cache(maxsize=4096)
def _lookup_grad_need(rows, width, t, to, table_rows):
    return _ripple.load_library().ripple_lookup_rows_grad_workspace_bytes(
        _LOOKUP_GRAD_ARGS.pack(rows, width, t, to, 0, 0, width, 0, 0, width, table_rows, 1.0, 0, 0, 0, 0))


@lru_cache(maxsize=4096)
def _norm_grad_need(rows, width, t, tx, vectors):
    return _ripple.load_library().ripple_norm_rows_grad_workspace_bytes(
        _NORM_GRAD_ARGS.pack(rows, width, t, tx, 0, 0, width, 0, width, rows, 0, 0, 0, 0, width, 64 if vectors else 0, 0, 1, 0.0, 0, 0, 0, 0, 0))


@lru_cache(maxsize=4096)
def _loss_need(rows, t, K, N, x_at, x_ld, w_at, w_ld):
    return _ripple.load_library().ripple_loss_rows_workspace_bytes(_LOSS_ARGS.pack(rows, t, K, N, 0, x_at, x_ld, w_at, w_ld, 0, 0, 0, 0, 0, 0, 0))


@lru_cache(maxsize=4096)
def _loss_grad_need(rows, t, K, N, x_at, x_ld, w_at, w_ld, dx_at, dw_at, bias):
    return _ripple.load_library().ripple_loss_rows_grad_workspace_bytes(_LOSS_GRAD_ARGS.pack(
        rows, t, K, N, 0, x_at, x_ld, w_at, w_ld, 0, 0, 0, 0, dx_at, K, dw_at, N, 64 if bias else 0, 1.0, 0, 0, 0, 0))


def _aligned_as(ptr: int) -> int:
    """An address that is not null and as aligned as this one."""
    return 1024 + (ptr & 255)


def _or_null(t) -> int:
    return 0 if t is None else t.data_ptr()


def lookup_rows(table, ids, scale: float = 1.0, out=None, out_dtype=None):
    """scale * table[ids], one row per id (int32), zeros for ids outside the table; formed in fp32.  The result has the table's type, or the one that
    out_dtype (or out) says if the table is fp32."""
    if getattr(forward_ad, "_current_level", 0) >= 0:
        _refuse_tangents(table=table, out=out)
    index = _device_of(table, "table")
    ptr, ld, table_rows = _matrix(table, "table", None, None, index)
    width = table.shape[1]
    ids_ptr, rows = _ids(ids, index)
    if out is None:
        out = torch.empty((rows, width), dtype=out_dtype or table.dtype, device=table.device)
        out_ptr, out_ld = out.data_ptr(), width
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out: {out_dtype} expected, got {out.dtype}")
        out_ptr, out_ld, got = _matrix(out, "out", width, None, index)
        if got != rows:
            raise ValueError(f"out: {rows} rows expected, got {got}")
    t, to = _type_of(table.dtype, "table"), _type_of(out.dtype, "out")
    if to != t and t != TYPE_F32:
        raise TypeError(f"out: {table.dtype} expected, got {out.dtype}")
    _check(_ripple.load_library().ripple_lookup_rows(_LOOKUP_ARGS.pack(
        rows, width, t, to, index, ptr, ld, table_rows, ids_ptr, out_ptr, out_ld, float(scale), 0, _stream(index))))
    return out


def lookup_rows_grad(dy, ids, table_rows: int, scale: float = 1.0, out=None, out_dtype=None, accumulate: bool = False):
    """The gradient of lookup_rows' table: [table_rows, D], row r = scale * the sum of dy's rows whose id is r; of dy's type, or fp32 if
    out_dtype (or out) says so.  accumulate: add to the rows of `out` that ids name, once for each, and touch no other."""
    if getattr(forward_ad, "_current_level", 0) >= 0:
        _refuse_tangents(dy=dy, out=out)
    index = _device_of(dy, "dy")
    ptr, ld, rows = _matrix(dy, "dy", None, None, index)
    width = dy.shape[1]
    ids_ptr, named = _ids(ids, index)
    if named != rows:
        raise ValueError(f"ids: {rows} entries expected, got {named}")
    if out is None:
        if accumulate:
            raise ValueError("accumulate without out")
        out = torch.empty((int(table_rows), width), dtype=out_dtype or dy.dtype, device=dy.device)
        out_ptr, out_ld = out.data_ptr(), width
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out: {out_dtype} expected, got {out.dtype}")
        out_ptr, out_ld, got = _matrix(out, "out", width, None, index)
        if got != table_rows:
            raise ValueError(f"out: {table_rows} rows expected, got {got}")
    t, to = _type_of(dy.dtype, "dy"), _type_of(out.dtype, "out")
    if to not in (t, TYPE_F32):
        raise TypeError(f"out: {dy.dtype} or float32 expected, got {out.dtype}")
    lib = _ripple.load_library()
    head = (rows, width, t, to, index, ptr, ld, ids_ptr, out_ptr, out_ld, int(table_rows), float(scale), bool(accumulate))
    need = _lookup_grad_need(rows, width, t, to, int(table_rows))
    work = _workspace(need, dy)
    _check(lib.ripple_lookup_rows_grad(_LOOKUP_GRAD_ARGS.pack(*head, _or_null(work), max(need, 0), _stream(index))))
    return out


def norm_rows_grad(dn, x, norm: Norm, ids=None, add=None, out=None, dx: bool = True, vectors: bool = True):
    """(dx, dweight, dbias) of n = norm(x[ids]) from dn [rows, D]; dweight and dbias (fp32) are None where the norm has no such
    vector, or with vectors=False; dx=False: no dx.  x [any, D]: dn's type or fp32; row ids[i] (int32) of it, or row i, was normalised.  dx [rows, D] has x's type; add [rows, D],
    of the same type: what reaches x past the norm, added before dx is rounded.  out: where to write dx; it may be dn, add, or, without ids, x."""
    if not isinstance(norm, Norm):
        raise TypeError(f"norm: a Norm expected, got {type(norm).__name__}")
    if getattr(forward_ad, "_current_level", 0) >= 0:
        _refuse_tangents(dn=dn, x=x, add=add, out=out)
    index = _device_of(dn, "dn")
    dn_ptr, dn_ld, rows = _matrix(dn, "dn", None, None, index)
    width = dn.shape[1]
    x_ptr, x_ld, x_rows = _matrix(x, "x", width, None, index)
    t, tx = _type_of(dn.dtype, "dn"), _type_of(x.dtype, "x")
    if tx not in (t, TYPE_F32):
        raise TypeError(f"x: {dn.dtype} or float32 expected, got {x.dtype}")
    ids_ptr = add_ptr = add_ld = 0
    if ids is not None:
        ids_ptr, named = _ids(ids, index)
        if named != rows:
            raise ValueError(f"ids: {rows} entries expected, got {named}")
    elif x_rows != rows:
        raise ValueError(f"x: {rows} rows expected, got {x_rows}")
    if add is not None:
        add_ptr, add_ld, got = _matrix(add, "add", width, x.dtype, index)
        if got != rows:
            raise ValueError(f"add: {rows} rows expected, got {got}")
    out_ptr, out_ld = 0, width
    if out is not None:
        if not dx:
            raise ValueError("out without dx")
        out_ptr, out_ld, got = _matrix(out, "out", width, x.dtype, index)
        if got != rows:
            raise ValueError(f"out: {rows} rows expected, got {got}")
    elif dx:
        out = torch.empty((rows, width), dtype=x.dtype, device=dn.device)
        out_ptr = out.data_ptr()
    dweight = torch.empty(width, dtype=torch.float32, device=dn.device) if vectors and norm.weight is not None else None
    dbias = torch.empty(width, dtype=torch.float32, device=dn.device) if vectors and norm.bias is not None else None
    if not dx and dweight is None and dbias is None:
        raise ValueError("no gradient wanted")
    lib = _ripple.load_library()
    stream = _stream(index)
    head = (rows, width, t, tx, index, dn_ptr, dn_ld, x_ptr, x_ld, x_rows, ids_ptr, add_ptr, add_ld, out_ptr, out_ld,
            _or_null(dweight), _or_null(dbias), *norm._packed(width, index, stream, "norm"))
    need = _norm_grad_need(rows, width, t, tx, dweight is not None or dbias is not None)
    work = _workspace(need, dn)
    _check(lib.ripple_norm_rows_grad(_NORM_GRAD_ARGS.pack(*head, _or_null(work), max(need, 0), stream)))
    return out, dweight, dbias


def _linear(x, W, labels, bias):
    """What both calls of the loss check of their inputs: sizes, addresses."""
    index = _device_of(x, "x")
    x_ptr, x_ld, rows = _matrix(x, "x", None, None, index)
    K = x.shape[1]
    w_ptr, w_ld, wk = _matrix(W, "W", None, x.dtype, index)
    if wk != K:
        raise ValueError(f"W: {K} rows expected, got {wk}")
    t = _type_of(x.dtype, "x")
    labels_ptr = _vector(labels, "labels", rows, torch.int32, index)
    bias_ptr = 0 if bias is None else _vector(bias, "bias", W.shape[1], torch.float32, index)
    N = W.shape[1]
    return index, rows, (rows, t, K, N, index, x_ptr, x_ld, w_ptr, w_ld, bias_ptr, labels_ptr), (rows, t, K, N, _aligned_as(x_ptr), x_ld, _aligned_as(w_ptr), w_ld)


def loss_rows(x, W, labels, bias=None):
    """(loss, lse), fp32 [rows]: lse_i = log sum_c exp z_ic, loss_i = lse_i - z_i,label with z = x W + bias; 0 for labels (int32) that are no
    class.  x [rows, K] and W [K, N] of one type, bias fp32; a bias of minus infinity takes a class out."""
    if getattr(forward_ad, "_current_level", 0) >= 0:
        _refuse_tangents(x=x, W=W, bias=bias)
    index, rows, head, sizes = _linear(x, W, labels, bias)
    device = x.device
    loss = torch.empty(rows, dtype=torch.float32, device=device)
    lse = torch.empty(rows, dtype=torch.float32, device=device)
    head = (*head, loss.data_ptr(), lse.data_ptr())
    lib = _ripple.load_library()
    need = _loss_need(*sizes)
    work = _workspace(need, x)
    _check(lib.ripple_loss_rows(_LOSS_ARGS.pack(*head, _or_null(work), max(need, 0), _stream(index))))
    return loss, lse


def loss_rows_grad(x, W, labels, lse, dloss=1.0, bias=None, dx: bool = True, dW: bool = True):
    """(dx, dW, dbias) of loss_rows, from what it gave as lse and dloss: fp32 [rows], or a number for all rows.  dx [rows, K] and
    dW [K, N] have the type of x and W (None where they are not wanted), dbias is fp32 (None without bias).  What each row adds is
    dloss_i (softmax(z)_i - onehot(label_i)): formed anew from x and W, in pieces of the classes."""
    if getattr(forward_ad, "_current_level", 0) >= 0:
        _refuse_tangents(x=x, W=W, bias=bias, lse=lse, dloss=dloss)
    index, rows, head, sizes = _linear(x, W, labels, bias)
    lse_ptr = _vector(lse, "lse", rows, torch.float32, index)
    scale, dloss_ptr = 1.0, 0
    if isinstance(dloss, torch.Tensor):
        dloss_ptr = _vector(dloss, "dloss", rows, torch.float32, index)
    else:
        scale = float(dloss)
    if not (dx or dW or bias is not None):
        raise ValueError("no gradient wanted")
    gx = torch.empty((rows, x.shape[1]), dtype=x.dtype, device=x.device) if dx else None
    gw = torch.empty(W.shape, dtype=W.dtype, device=x.device) if dW else None
    gb = torch.empty(W.shape[1], dtype=torch.float32, device=x.device) if bias is not None else None
    head = (*head, lse_ptr, dloss_ptr, _or_null(gx), x.shape[1], _or_null(gw), W.shape[1], _or_null(gb), scale, 0)
    lib = _ripple.load_library()
    need = _loss_grad_need(*sizes, _aligned_as(gx.data_ptr()) if dx else 0, _aligned_as(gw.data_ptr()) if dW else 0, bias is not None)
    work = _workspace(need, x)
    _check(lib.ripple_loss_rows_grad(_LOSS_GRAD_ARGS.pack(*head, _or_null(work), max(need, 0), _stream(index))))
    return gx, gw, gb


class LiveNorm(Norm):
    """A norm whose vectors are the caller's own tensors (fp32, CUDA), `weight` and `bias`: what is written into them, and what is put in their
    place, is seen by the next call."""

    def __init__(self, kind: int, weight, bias=None, eps: float = 1e-5):
        if kind not in (NORM_LAYER, NORM_RMS):
            raise ValueError(f"kind: NORM_LAYER or NORM_RMS expected, got {kind}")
        if not eps >= 0:
            raise ValueError(f"eps: {eps}")
        index = _device_of(weight, "weight")
        if weight.dim() != 1:
            raise ValueError(f"weight: one dimension expected, got {tuple(weight.shape)}")
        self.kind, self.eps, self.weight, self.bias = int(kind), float(eps), weight, bias
        self._at = None
        self._packed(weight.shape[0], index, _stream(index), "norm")

    @property
    def width(self):
        return self.weight.shape[0]

    @property
    def index(self):
        return self.weight.get_device()

    def _packed(self, width: int, index: int, stream: int, name: str):
        weight, bias = self.weight, self.bias
        at = _vector(weight, name + ": weight", width, torch.float32, index), 0 if bias is None else _vector(bias, name + ": bias", width, torch.float32, index)
        if at != self._at:           # (other memory than at the call before: no stream is known to read it yet)
            self._keep(None, *(t for t in (weight, bias) if t is not None))
            self._at = at
        self._read_on(stream)
        return self.kind, self.eps, *at


class ClassHead:
    """Classes of vertices from their cached rows:  logits = norm(table[ids] + scale * E[kinds]) W + bias.

    Parameters, CUDA tensors that an optimiser updates in place or others of their shape and type take the place of: `norm_weight`, `norm_bias` (fp32 [D]; no bias for NORM_RMS), `W` [D, N] of
    `dtype`, `bias` (fp32 [N]), and, with `kinds` > 0, `E` [kinds, D] of `dtype`: learned rows of what a vertex is, beside what the graph's layers
    made of it.  W is drawn from N(0, 1 / D), E starts at zero."""

    def __init__(self, D: int, N: int, kinds: int = 0, kind: int = NORM_LAYER, eps: float = 1e-5, scale: float = 1.0, dtype=torch.float32,
                 device=None, seed: int = 0):
        _type_of(dtype, "dtype")
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        f32 = dict(dtype=torch.float32, device=device)            # (whatever PyTorch's default type is)
        self.W = (torch.randn(D, N, generator=torch.Generator(device=device).manual_seed(seed), **f32) * D ** -0.5).to(dtype)
        self.bias = torch.zeros(N, **f32)
        self.E = torch.zeros(kinds, D, dtype=dtype, device=device) if kinds > 0 else None
        self.scale = float(scale)
        self.norm = LiveNorm(kind, torch.ones(D, **f32), torch.zeros(D, **f32) if kind == NORM_LAYER else None, eps)

    norm_weight = property(lambda self: self.norm.weight, lambda self, t: setattr(self.norm, "weight", t))
    norm_bias = property(lambda self: self.norm.bias, lambda self, t: setattr(self.norm, "bias", t))

    def parameters(self) -> Dict[str, torch.Tensor]:
        """The parameters by name, as the gradients are."""
        return {k: t for k, t in (("norm_weight", self.norm_weight), ("norm_bias", self.norm_bias), ("W", self.W), ("bias", self.bias), ("E", self.E))
                if t is not None}

    def _live(self, table, ids, labels):
        """ids, rows and labels of the rows that take part; -1 in all three for the others."""
        index = _device_of(table, "table")
        table_rows = _matrix(table, "table", None, None, index)[2]
        ids_ptr, rows = _ids(ids, index)
        labels_ptr = _vector(labels, "labels", rows, torch.int32, index)
        live = torch.empty((3, rows), dtype=torch.int32, device=table.device)
        at = live.data_ptr()
        _check(_ripple.load_library().ripple_live_rows(_LIVE_ARGS.pack(
            rows, self.W.shape[1], index, ids_ptr, table_rows, labels_ptr, at, at + 4 * rows, at + 8 * rows, _stream(index))))
        return live.unbind(0)

    def _normed(self, table, ids, kinds):
        """The rows before the norm (None: the table's own) and behind it."""
        if (kinds is None) != (self.E is None):
            raise ValueError("kinds go with the learned rows: the head has " + ("none" if self.E is None else "some"))
        if self.E is None:
            return None, norm_rows(residual=table, ids=ids, pre=self.norm, normed_dtype=self.W.dtype, clear_padding=True)[1]
        return norm_rows(lookup_rows(self.E, kinds, self.scale), residual=table, ids=ids, pre=self.norm, clear_padding=True)

    def loss(self, table, ids, labels, kinds=None):
        """The losses of the rows `ids` (int32) of `table` (fp32, or the head's type), fp32 [len(ids)]; 0 where the id names no row or the
        label (int32) no class."""
        ids, _, labels = self._live(table, ids, labels)
        return loss_rows(self._normed(table, ids, kinds)[1], self.W, labels, self.bias)[0]

    def step(self, table, ids, labels, kinds=None, dloss=1.0):
        """(loss, gradients): the losses as `loss` gives them, and by parameter the gradient of their sum weighted by dloss (a number, or
        fp32 [len(ids)]).  Rows whose id names no row of the table or whose label no class (-1 by custom) have loss 0 and add nothing to any gradient, whatever the
        table and dloss hold there; kinds out of range are vertices without a learned row.  Gradients have the shape and type of their parameter (E's is summed in fp32)."""
        ids, rows, labels = self._live(table, ids, labels)
        s, n = self._normed(table, ids, kinds)
        loss, lse = loss_rows(n, self.W, labels, self.bias)
        dn, dW, dbias = loss_rows_grad(n, self.W, labels, lse, dloss, self.bias)
        if s is None:
            ds, dweight, dnorm_bias = norm_rows_grad(dn, table, self.norm, ids=ids, dx=False)
        else:
            ds, dweight, dnorm_bias = norm_rows_grad(dn, s, self.norm, ids=rows)
        got = {"norm_weight": dweight, "W": dW, "bias": dbias}
        if dnorm_bias is not None:
            got["norm_bias"] = dnorm_bias
        if self.E is not None:
            got["E"] = lookup_rows_grad(ds, kinds, self.E.shape[0], self.scale).to(self.E.dtype)
        return loss, got

    def request_head(self) -> RequestHead:
        """What requests run: the head's norm and linear layer as they are now (copies).  Heads with learned rows have no such form."""
        if self.E is not None:
            raise ValueError("a head with learned rows has no form for requests")
        return RequestHead([], Norm(self.norm.kind, self.norm_weight, self.norm_bias, self.norm.eps), Projection(self.W, self.bias))
