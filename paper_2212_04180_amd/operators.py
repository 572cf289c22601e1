"""Operators of networks over torch tensors (es_dense, es_gated, their
gradients and es_adamw of include/esmi.h).

For programs with a network of their own beside the strategies: the layers of
a population's networks -- w[n] a view into member n of es.ask(materialize=
True), cast where it is to run in 16 bits -- or of one network, their gradients,
and an optimiser step outside es_tell.  Argument marshalling only, as in
esmi.py; outputs and workspaces come from torch's allocator on the stream that
the kernels run on.  Nothing is recorded by autograd: the gradients are calls
of their own, and where autograd records (outside torch.no_grad()) the layers
refuse operands that require a gradient.
"""
from __future__ import annotations

import ctypes
import math
import struct
from itertools import chain

import torch
from torch.autograd.graph import increment_version  # autograd then knows a tensor that it saved as changed

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


def _check(rc):
    if rc != esmi.ES_OK:
        raise EsError(rc, esmi.lib().es_last_error(None).decode())


def _launch(name, packed, device):
    """The call on the device's current stream; most need no workspace, so that its size is asked for only where the
    call without one was refused (a microsecond of a small call's ten)."""
    if torch.cuda.current_device() != device:
        with torch.cuda.device(device):
            return _launch(name, packed, device)
    lib, stream = esmi.lib(), _stream(device)
    rc = getattr(lib, name)(packed, None, 0, stream)
    if rc != esmi.ES_ERR_ARG:  # done, or failed with something perhaps enqueued
        _check(rc)
        return
    n = ctypes.c_size_t(0)
    _check(getattr(lib, name + "_workspace")(packed, ctypes.byref(n)))
    if n.value == 0:  # refused for something else
        _check(getattr(lib, name)(packed, None, 0, stream))
        return
    ws = torch.empty(n.value, dtype=torch.uint8, device=device)
    _check(getattr(lib, name)(packed, ws.data_ptr(), n.value, stream))


def _stream(device):
    """torch.cuda.current_stream(device).cuda_stream, without the Stream object: 2 us less of a call's 12."""
    return torch._C._cuda_getCurrentRawStream(device)


def _matrix(name, t, dtype, device, rows, cols):
    """(pointer, member stride, row stride), rows, cols and members (None: the same for all).  rows, cols: the size
    expected (None: any)."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not dtype or t.get_device() != device:
        _place(name, t, dtype, device)
    if t.requires_grad and torch.is_grad_enabled():
        _unrecorded(name)
    if len(shape) == 2:
        (r, c), (row, one), member, n = shape, stride, 0, None
    elif len(shape) == 3:
        (n, r, c), (member, row, one) = shape, stride
    else:
        raise ValueError(f"{name} has {len(shape)} dimensions, not 2 or, with members, 3")
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise ValueError(f"{name} is {tuple(shape)}, expected {rows} x {cols}")
    if one != 1 and c > 1:
        raise ValueError(f"{name}: the elements of a row must follow each other")
    return (t.data_ptr(), member, row), r, c, n


def _vector(name, t, dtype, device, n, members):
    """The bias, with members exactly where w has them."""
    shape = t.shape
    if t.dtype is not dtype or t.get_device() != device:
        _place(name, t, dtype, device)
    if t.requires_grad and torch.is_grad_enabled():
        _unrecorded(name)
    if len(shape) not in (1, 2):
        raise ValueError(f"{name} has {len(shape)} dimensions, not 1 or, with members, 2")
    if shape[-1] != n:
        raise ValueError(f"{name} has {shape[-1]} elements, not {n}")
    if (len(shape) == 1) != (members is None) or (members is not None and shape[0] != members):
        raise ValueError(f"{name} must have members exactly where w has")
    if n > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a row must follow each other")
    return t.data_ptr(), t.stride(0) if members is not None else 0, 0


def _place(name, t, dtype, device):
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{device}")
    raise ValueError(f"{name} is {t.dtype}, not {dtype}")


def _unrecorded(name):
    raise ValueError(f"{name} requires a gradient, and autograd does not record this call: under torch.no_grad(), or "
                     f"detached, with the gradient from the _backward call")


def _first(t):
    """Type and device that the other operands share."""
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if t.dtype not in _DTYPES:
        raise ValueError(f"fp32, bf16 or fp16 expected, not {t.dtype}")
    return t.dtype, t.get_device()


def _overlap(a, b):
    """Whether matrices (of members) may share memory.  False only where they do not: their ranges are apart, or they
    lie between each other's members or rows, which then repeat at common multiples."""
    if a.numel() == 0 or b.numel() == 0:
        return False
    first = [t.data_ptr() for t in (a, b)]
    steps = [[(n - 1, s * t.element_size()) for n, s in zip(t.shape, t.stride())] for t in (a, b)]

    def span(dims, t):  # bytes from the first element of these dimensions to behind the last
        return sum(n * s for n, s in dims) + t.element_size()

    d = first[1] - first[0]
    if d >= span(steps[0], a) or -d >= span(steps[1], b):
        return False
    for inner in (1, 2):  # dimensions of a block: a row, a member's matrix
        every = math.gcd(*(s for dims in steps for n, s in dims[:-inner] if n))
        if every and d % every >= span(steps[0][-inner:], a) and d % every + span(steps[1][-inner:], b) <= every:
            return False
    return True


def _apart(out, x, w, bias, residual):
    """out receives results while the operands are still read: only the residual's own elements are read by who writes
    them."""
    for name, t in (("x", x), ("w", w), ("bias", bias.unsqueeze(-2) if bias is not None else None)):
        if t is not None and _overlap(out, t):
            raise ValueError(f"out shares memory with {name}")
    if residual is None or (out.data_ptr() == residual.data_ptr() and out.dtype is residual.dtype and
                            [(n, s) for n, s in zip(out.shape, out.stride()) if n > 1] ==
                            [(n, s) for n, s in zip(residual.shape, residual.stride()) if n > 1]):
        return
    if _overlap(out, residual):
        raise ValueError("out shares memory with the residual, but is not the residual itself")


def _members(named):
    """The one count of members among operands, None: none has any."""
    n = None
    for name, m in named:
        if m is not None and m != n:
            if n is not None:
                raise ValueError(f"{name} has {m} members, not {n}")
            n = m
    return n


def _shape(members, *sizes):
    return sizes if members is None else (members, *sizes)


def _act(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"unknown activation {name!r}: one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[name]


def _forward(entry, gated, x, w, bias, residual, act, keep_pre, out_dtype, out):
    dt, dev = _first(x)
    px, rows, k, nx = _matrix("x", x, dt, dev, None, None)
    pw, wide, _, nw = _matrix("w", w, dt, dev, None, k)
    if gated and wide % 2:
        raise ValueError(f"w of a gated layer has an even number of rows, gates first: not {wide}")
    f = wide // 2 if gated else wide
    pb = _vector("bias", bias, dt, dev, wide, nw) if bias is not None else _NONE
    pr, nr = _NONE, None
    if residual is not None:
        pr, _, _, nr = _matrix("residual", residual, dt, dev, rows, f)
    n = _members((("x", nx), ("w", nw), ("residual", nr)))
    if out is None:
        y, ydt = None, out_dtype or dt
    else:
        y, ydt = out, out.dtype
        if out_dtype is not None and ydt is not out_dtype:
            raise ValueError(f"the output is {ydt}, not {out_dtype}")
    if ydt is not dt and ydt is not torch.float32:
        raise ValueError(f"the output is {dt} or fp32, not {ydt}")
    if y is None:
        y = torch.empty(_shape(n, rows, f), dtype=ydt, device=dev)
        py = y.data_ptr(), rows * f, f
    else:
        py, _, _, ny = _matrix("out", y, ydt, dev, rows, f)
        if ny != n:
            raise ValueError("out has members exactly where an operand has")
        _apart(out, x, w, bias, residual)
    pre, pp = None, _NONE
    if keep_pre:
        pre = torch.empty(_shape(n, rows, wide), dtype=dt, device=dev)
        pp = pre.data_ptr(), rows * wide, wide
    packed = _FORWARD.pack(_DTYPES[dt], _DTYPES[ydt], _act(act), 0, 1 if n is None else n, rows, k, f,
                           *px, *pw, *pb, *pr, *py, *pp)
    _launch(entry, packed, dev)
    if out is not None:
        increment_version(out)
    return (y, pre) if keep_pre else y


def _backward(entry, gated, dy, x, w, pre, act, needs):
    dt, dev = _first(dy)
    pd, rows, f, n = _matrix("dy", dy, dt, dev, None, None)
    wide = 2 * f if gated else f
    px, _, k, nx = _matrix("x", x, dt, dev, rows, None)
    pw, _, _, nw = _matrix("w", w, dt, dev, wide, k)
    pp, npre = _NONE, None
    if pre is not None:
        pp, _, _, npre = _matrix("pre", pre, dt, dev, rows, wide)
    elif gated or act != "none":
        raise ValueError("pre is needed: the forward keeps it with keep_pre=True")
    if _members((("dy", n), ("x", nx), ("w", nw), ("pre", npre))) != n:
        raise ValueError("dy has no members, but another operand has")
    need_x, need_w, need_b = needs
    dx = torch.empty(_shape(nx, rows, k), dtype=dt, device=dev) if need_x else None
    dw = torch.empty(_shape(nw, wide, k), dtype=dt, device=dev) if need_w else None
    db = torch.empty(_shape(nw, wide), dtype=dt, device=dev) if need_b else None
    packed = _BACKWARD.pack(_DTYPES[dt], _act(act), 1 if n is None else n, rows, k, f, *pd, *px, *pw, *pp,
                            *((dx.data_ptr(), 0 if nx is None else rows * k, k) if need_x else _NONE),
                            *((dw.data_ptr(), 0 if nw is None else wide * k, k) if need_w else _NONE),
                            *((db.data_ptr(), 0 if nw is None else wide, 0) if need_b else _NONE))
    _launch(entry, packed, dev)
    return dx, dw, db


def _on(stream, tensors, f, *args):
    """f on that stream.  It first waits for the current one, where the operands may still be being made, and they are
    marked as in use there: a temporary freed on return is not handed out again before the kernels have passed."""
    if stream is None:
        return f(*args)
    for t in tensors:
        if t is not None and t.is_cuda and t.device != stream.device:
            raise ValueError(f"the stream is on {stream.device}, an operand on {t.device}")
    here = torch.cuda.current_stream(stream.device)
    if stream == here:
        return f(*args)
    stream.wait_stream(here)
    for t in tensors:
        if t is not None and t.is_cuda:
            t.record_stream(stream)
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
    takes.  out: where y goes; may be the residual itself, but share memory with
    nothing else.  stream: None, the current one."""
    return _on(stream, (x, w, bias, residual, out), _forward, "es_dense", False, x, w, bias, residual, act, keep_pre, out_dtype, out)


def dense_backward(dy, x, w, pre=None, act="none", needs=(True, True, True), stream=None):
    """(dx, dw, db) of dense for dy = dL/dy (the residual's gradient is dy, or
    dy.sum(0) where the members share it), shaped like x, w and the bias: an
    operand without members in a call with members receives the sum over them.
    needs: which to compute, None for the others.  dz = dy act'(pre) takes the
    type's precision and range before the products dx = dz w and dw = dz^T x;
    db sums it unrounded."""
    return _on(stream, (dy, x, w, pre), _backward, "es_dense_backward", False, dy, x, w, pre, act, needs)


def gated(x, w, bias=None, act="silu", keep_pre=False, out_dtype=None, out=None, stream=None):
    """h = act(g) u with [g, u] = x w^T + bias: w [2 out, in], the gates' rows
    first.  The first half of a gated feed-forward block; the second is
    dense(h, w_down, residual=x).  Shapes, types and strides as in dense; pre
    is [g, u], ([members,] rows, 2 out)."""
    return _on(stream, (x, w, bias, out), _forward, "es_gated", True, x, w, bias, None, act, keep_pre, out_dtype, out)


def gated_backward(dh, x, w, pre, act="silu", needs=(True, True, True), stream=None):
    """(dx, dw, db) of gated for dh = dL/dh; see dense_backward."""
    return _on(stream, (dh, x, w, pre), _backward, "es_gated_backward", True, dh, x, w, pre, act, needs)


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
        if t.dtype is not dtype or t.get_device() != device:
            raise ValueError(f"{name} must be {dtype} on cuda:{device}, not {t.dtype} on {t.device}")
        if t.numel() != size or not t.is_contiguous():
            raise ValueError(f"{name}: contiguous tensors of the parameters' sizes expected")
    return [t.data_ptr() for t in ts]


def _distinct(cols, sizes, bits, copied):
    """What is written is written for one tensor only, and is no gradient."""
    lists = [0, 2, 3] + ([4, 5] if bits == 8 else []) + ([6] if copied else [])
    flat = list(chain.from_iterable(cols[i] for i in lists))
    seen = set(flat)
    if len(seen) == len(flat) and seen.isdisjoint(cols[1]):
        return
    # empty tensors may lie anywhere
    flat = [p for i in lists for p, k in zip(cols[i], sizes) if k]
    seen = set(flat)
    if len(seen) != len(flat):
        raise ValueError("a parameter, state, scale or copy is listed twice")
    if not seen.isdisjoint(p for p, k in zip(cols[1], sizes) if k):
        raise ValueError("a gradient is also a parameter, state, scale or copy")


def adamw(params, grads, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, m_scale=None, v_scale=None,
          copies=None, stream=None):
    """One AdamW step (step >= 1) on lists of tensors, in place, in few launches.

    params fp32; grads fp32, bf16 or fp16.  m, v: fp32, or float8_e4m3fn with
    m_scale, v_scale (adamw_state makes either): m and the square root of v as
    codes, one fp32 scale per 256 elements.  copies: bf16 or fp16 tensors that
    receive the new parameters.  lr, weight_decay: numbers, or one per tensor.
    All contiguous, none overlapping another.  A captured call repeats its
    step number.  stream: as in dense."""
    if stream is not None:
        tensors = [t for ts in (params, grads, m, v, m_scale, v_scale, copies) if ts is not None for t in ts]
        return _on(stream, tensors, adamw, params, grads, m, v, step, lr, beta1, beta2, eps, weight_decay, m_scale, v_scale, copies)
    n = len(params)
    if n == 0:
        return
    if not params[0].is_cuda:
        raise ValueError("device tensor expected")
    device = params[0].get_device()
    if torch.cuda.current_device() != device:
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
        each = [float(e) for e in value] if isinstance(value, (list, tuple)) else [float(value)] * n
        if len(each) != n:
            raise ValueError(f"{name}: one number, or one per parameter")
        cols.append(each)
    _distinct(cols, sizes, bits, copies is not None)
    table = struct.pack("=" + _TENSOR * n, *chain.from_iterable(zip(*cols)))
    head = _ADAMW.pack(n, _DTYPES[gdt], bits, _DTYPES[cdt], int(step), beta1, beta2, eps, 0)
    _check(esmi.lib().es_adamw(head, table, _stream(device)))
    increment_version([*params, *m, *v, *(t for ts in (copies, m_scale, v_scale) if ts is not None for t in ts)])
