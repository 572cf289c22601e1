"""Operators of networks over torch tensors (es_dense, es_gated, their
gradients and es_adamw of include/esmi.h).

For programs with a network of their own beside the strategies: the layers of
a population's networks -- w[n] a view into member n of es.ask(materialize=
True), cast where it is to run in 16 bits -- or of one network, their gradients,
and an optimiser step outside es_tell.  Argument marshalling only, as in
esmi.py; outputs and workspaces come from torch's allocator on the stream that
the kernels run on.  Nothing is recorded by autograd: the gradients are calls
of their own.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import esmi
from .esmi import EsError

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "tanh": 2, "gelu": 3, "silu": 4}
_F8 = torch.float8_e4m3fn
_BLOCK = 256  # elements that share a scale of adamw's 8-bit states

_FORWARD = struct.Struct("=iiiiqqqq" + "Qqq" * 6)   # es_dense_args
_BACKWARD = struct.Struct("=iiqqqq" + "Qqq" * 7)    # es_dense_grad_args
_TENSOR = "QQQQQQQqff"                              # es_adamw_tensor
_ADAMW = struct.Struct("=iiiiqfffi")                # es_adamw_args
_NONE = (0, 0, 0)


def _call(name, *args):
    rc = getattr(esmi.lib(), name)(*args)
    if rc != esmi.ES_OK:
        raise EsError(rc, esmi.lib().es_last_error(None).decode())


def _launch(name, packed, device):
    """Workspace from the query, then the call on the device's current stream."""
    if torch.cuda.current_device() != device.index:
        with torch.cuda.device(device):
            return _launch(name, packed, device)
    n = ctypes.c_size_t(0)
    _call(name + "_workspace", packed, ctypes.byref(n))
    ws = torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None
    _call(name, packed, ws.data_ptr() if ws is not None else None, n.value, torch.cuda.current_stream(device).cuda_stream)


class _Shapes:
    """Collects the operands' member counts and makes their (pointer, member stride, row stride)."""

    def __init__(self, like):
        if not like.is_cuda:
            raise ValueError("device tensor expected")
        if like.dtype not in _DTYPES:
            raise ValueError(f"fp32, bf16 or fp16 expected, not {like.dtype}")
        self.dtype, self.device, self.members = like.dtype, like.device, None

    def _look(self, name, t, dims, dtype):
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, not on {self.device}")
        if t.dtype != (dtype or self.dtype):
            raise ValueError(f"{name} is {t.dtype}, not {dtype or self.dtype}")
        if t.dim() not in (dims, dims + 1):
            raise ValueError(f"{name} has {t.dim()} dimensions, not {dims} or, with members, {dims + 1}")
        if t.dim() == dims + 1:
            if self.members is None:
                self.members = t.shape[0]
            elif self.members != t.shape[0]:
                raise ValueError(f"{name} has {t.shape[0]} members, not {self.members}")
        if t.stride(-1) != 1 and t.shape[-1] > 1:
            raise ValueError(f"{name}: the elements of a row must follow each other")

    def matrix(self, name, t, rows, cols, dtype=None):
        """rows and cols: the size expected (None: any).  A 2-D tensor is the same for all members."""
        self._look(name, t, 2, dtype)
        if (rows is not None and t.shape[-2] != rows) or (cols is not None and t.shape[-1] != cols):
            raise ValueError(f"{name} is {tuple(t.shape)}, expected {rows} x {cols}")
        st = t.stride()
        return (t.data_ptr(), st[0], st[1]) if t.dim() == 3 else (t.data_ptr(), 0, st[0])

    def vector(self, name, t, n, members):
        if t is None:
            return _NONE
        self._look(name, t, 1, None)
        if t.shape[-1] != n:
            raise ValueError(f"{name} has {t.shape[-1]} elements, not {n}")
        if (t.dim() == 2) != members:
            raise ValueError(f"{name} must have members exactly where w has")
        return (t.data_ptr(), t.stride(0) if members else 0, 0)

    def empty(self, rows, cols, members, dtype=None):
        shape = (self.members, rows, cols) if members else (rows, cols)
        return torch.empty(shape, dtype=dtype or self.dtype, device=self.device)


def _act(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"unknown activation {name!r}: one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[name]


def _forward(entry, gated, x, w, bias, residual, act, keep_pre, out_dtype, out):
    s = _Shapes(x)
    px = s.matrix("x", x, None, None)
    rows, k = x.shape[-2:]
    pw = s.matrix("w", w, None, k)
    wide = w.shape[-2]
    if gated and wide % 2:
        raise ValueError(f"w of a gated layer has an even number of rows, gates first: not {wide}")
    f = wide // 2 if gated else wide
    pb = s.vector("bias", bias, wide, w.dim() == 3)
    pr = s.matrix("residual", residual, rows, f) if residual is not None else _NONE
    members = s.members is not None
    ydt = out_dtype or (out.dtype if out is not None else s.dtype)
    if ydt not in (s.dtype, torch.float32):
        raise ValueError(f"the output is {s.dtype} or fp32, not {ydt}")
    y = out if out is not None else s.empty(rows, f, members, ydt)
    if y.dim() != 2 + members:
        raise ValueError("out has members exactly where an operand has")
    py = s.matrix("out", y, rows, f, ydt)
    pre = s.empty(rows, wide, members) if keep_pre else None
    pp = s.matrix("pre", pre, rows, wide) if keep_pre else _NONE
    packed = _FORWARD.pack(_DTYPES[s.dtype], _DTYPES[ydt], _act(act), 0, s.members if members else 1, rows, k, f,
                           *px, *pw, *pb, *pr, *py, *pp)
    _launch(entry, packed, s.device)
    return (y, pre) if keep_pre else y


def _backward(entry, gated, dy, x, w, pre, act, needs):
    s = _Shapes(dy)
    pd = s.matrix("dy", dy, None, None)
    rows, f = dy.shape[-2:]
    wide = 2 * f if gated else f
    px = s.matrix("x", x, rows, None)
    k = x.shape[-1]
    pw = s.matrix("w", w, wide, k)
    if pre is None and (gated or act != "none"):
        raise ValueError("pre is needed: the forward keeps it with keep_pre=True")
    pp = s.matrix("pre", pre, rows, wide) if pre is not None else _NONE
    members = s.members is not None
    if members and dy.dim() != 3:
        raise ValueError("dy has no members, but another operand has")
    need_x, need_w, need_b = needs
    dx = s.empty(rows, k, x.dim() == 3) if need_x else None
    dw = s.empty(wide, k, w.dim() == 3) if need_w else None
    db = torch.empty((s.members, wide) if w.dim() == 3 else (wide,), dtype=s.dtype, device=s.device) if need_b else None
    packed = _BACKWARD.pack(_DTYPES[s.dtype], _act(act), s.members if members else 1, rows, k, f, *pd, *px, *pw, *pp,
                            *(s.matrix("dx", dx, rows, k) if need_x else _NONE),
                            *(s.matrix("dw", dw, wide, k) if need_w else _NONE),
                            *(s.vector("db", db, wide, w.dim() == 3) if need_b else _NONE))
    _launch(entry, packed, s.device)
    return dx, dw, db


def _on(stream, f, *args):
    if stream is None:
        return f(*args)
    with torch.cuda.stream(stream):
        return f(*args)


def dense(x, w, bias=None, residual=None, act="none", keep_pre=False, out_dtype=None, out=None, stream=None):
    """y = act(x w^T + bias) + residual.

    x [rows, in], w [out, in], bias [out], residual [rows, out]; any of them
    with a leading dimension of members (the bias exactly where w has it),
    the others are then the same for all.  One type, fp32, bf16 or fp16; sums
    in fp32.  Any strides whose rows are contiguous.  act: none, relu, tanh,
    gelu (erf form) or silu.  Returns y ([members,] rows, out) in the type, or
    fp32 with out_dtype; with keep_pre also x w^T + bias, which the gradient
    takes.  out: where y goes; may be the residual itself.  stream: None, the
    current one."""
    return _on(stream, _forward, "es_dense", False, x, w, bias, residual, act, keep_pre, out_dtype, out)


def dense_backward(dy, x, w, pre=None, act="none", needs=(True, True, True), stream=None):
    """(dx, dw, db) of dense for dy = dL/dy (the residual's gradient is dy),
    shaped like x, w and the bias: an operand without members in a call with
    members receives the sum over them.  needs: which to compute, None for the
    others."""
    return _on(stream, _backward, "es_dense_backward", False, dy, x, w, pre, act, needs)


def gated(x, w, bias=None, act="silu", keep_pre=False, out_dtype=None, out=None, stream=None):
    """h = act(g) u with [g, u] = x w^T + bias: w [2 out, in], the gates' rows
    first.  The first half of a gated feed-forward block; the second is
    dense(h, w_down, residual=x).  Shapes, types and strides as in dense; pre
    is [g, u], ([members,] rows, 2 out)."""
    return _on(stream, _forward, "es_gated", True, x, w, bias, None, act, keep_pre, out_dtype, out)


def gated_backward(dh, x, w, pre, act="silu", needs=(True, True, True), stream=None):
    """(dx, dw, db) of gated for dh = dL/dh; see dense_backward."""
    return _on(stream, _backward, "es_gated_backward", True, dh, x, w, pre, act, needs)


def adamw_state(params, bits=32):
    """Zero states of adamw for these parameters: dict of m, v and, with 8
    bits, m_scale and v_scale."""
    if bits not in (8, 32):
        raise ValueError("states have 32 or 8 bits")
    if bits == 32:
        return {k: [torch.zeros_like(p, memory_format=torch.contiguous_format) for p in params] for k in ("m", "v")}
    s = {k: [torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(_F8) for p in params] for k in ("m", "v")}
    for k in ("m_scale", "v_scale"):
        s[k] = [torch.zeros(-(-p.numel() // _BLOCK), dtype=torch.float32, device=p.device) for p in params]
    return s


def _tensors(name, ts, n, dtype, device, sizes):
    """Pointers of a list that goes with the parameters."""
    if len(ts) != n:
        raise ValueError(f"{name} has {len(ts)} tensors for {n} parameters")
    for t, size in zip(ts, sizes):
        if t.dtype is not dtype or t.device != device:
            raise ValueError(f"{name} must be {dtype} on {device}, not {t.dtype} on {t.device}")
        if t.numel() != size or not t.is_contiguous():
            raise ValueError(f"{name}: contiguous tensors of the parameters' sizes expected")
    return [t.data_ptr() for t in ts]


def adamw(params, grads, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, m_scale=None, v_scale=None,
          copies=None, stream=None):
    """One AdamW step (step >= 1) on lists of tensors, in place, in few launches.

    params fp32; grads fp32, bf16 or fp16.  m, v: fp32, or float8_e4m3fn with
    m_scale, v_scale (adamw_state makes either): m and the square root of v as
    codes, one fp32 scale per 256 elements.  copies: bf16 or fp16 tensors that
    receive the new parameters.  lr, weight_decay: numbers, or one per tensor.
    All contiguous, none overlapping another.  A captured call repeats its
    step number."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return adamw(params, grads, m, v, step, lr, beta1, beta2, eps, weight_decay, m_scale, v_scale, copies)
    n = len(params)
    if n == 0:
        return
    if not params[0].is_cuda:
        raise ValueError("device tensor expected")
    device = params[0].device
    if torch.cuda.current_device() != device.index:
        with torch.cuda.device(device):
            return adamw(params, grads, m, v, step, lr, beta1, beta2, eps, weight_decay, m_scale, v_scale, copies)
    sizes = [p.numel() for p in params]
    if len(grads) != n or len(m) != n:
        raise ValueError(f"{len(grads)} gradients and {len(m)} states for {n} parameters")
    gdt, sdt = grads[0].dtype, m[0].dtype
    if gdt not in _DTYPES:
        raise ValueError(f"gradients are fp32, bf16 or fp16, not {gdt}")
    if sdt not in (torch.float32, _F8):
        raise ValueError(f"states are fp32 or float8_e4m3fn, not {sdt}")
    bits = 32 if sdt is torch.float32 else 8
    cols = [_tensors("params", params, n, torch.float32, device, sizes), _tensors("grads", grads, n, gdt, device, sizes),
            _tensors("m", m, n, sdt, device, sizes), _tensors("v", v, n, sdt, device, sizes)]
    if len(set(cols[0])) != n and len({p for p, k in zip(cols[0], sizes) if k}) != sum(k > 0 for k in sizes):
        raise ValueError("a parameter is listed twice")
    if bits == 8:
        if m_scale is None or v_scale is None:
            raise ValueError("8-bit states need m_scale and v_scale")
        blocks = [-(-k // _BLOCK) for k in sizes]
        cols += [_tensors("m_scale", m_scale, n, torch.float32, device, blocks),
                 _tensors("v_scale", v_scale, n, torch.float32, device, blocks)]
    else:
        cols += [[0] * n, [0] * n]
    cdt = torch.bfloat16
    if copies is not None and len(copies):
        cdt = copies[0].dtype
        if cdt not in (torch.bfloat16, torch.float16):
            raise ValueError(f"copies are bf16 or fp16, not {cdt}")
    cols.append(_tensors("copies", copies, n, cdt, device, sizes) if copies is not None else [0] * n)
    cols.append(sizes)
    for name, value in (("lr", lr), ("weight_decay", weight_decay)):
        each = [float(value)] * n if isinstance(value, (int, float)) else [float(e) for e in value]
        if len(each) != n:
            raise ValueError(f"{name}: one number, or one per parameter")
        cols.append(each)
    table = struct.pack("=" + _TENSOR * n, *(e for row in zip(*cols) for e in row))
    head = _ADAMW.pack(n, _DTYPES[gdt], bits, _DTYPES[cdt], int(step), beta1, beta2, eps, 0)
    _call("es_adamw", head, table, torch.cuda.current_stream(device).cuda_stream)
