"""Plain 64-bit forms of the layer operators and the bounds of their errors.

Bounds, elementwise (u = 2^-24, h = eps_T / 2 the half step of the type T):
  z     sums of K products in fp32 in any order: K u sum|x||w|, the bias's
        addition u |z|
  act   every activation here has a slope of at most 1.13, and its fp32 value
        is within 16 u (|z| + 1) of the true one (libm-grade functions, a few
        roundings; z - its sum's error - moves it by at most 1.13 of it)
  y     rounded once: h |y|, or half the spacing of fp16's subnormals, 2^-25
  dz    dy times a slope within 16 u (3 for its conditioning): rounded to T
        before the products: h |dz|, 2^-25; slopes of a kept pre are taken at
        that pre, so its rounding is no error
  dx,dw sums over K terms of dz and an exact operand
  db    fp32 within a chunk of rows, fp64 between: (64 + 4) u sum|dz|
"""
import math

import torch

U = 2.0 ** -24
SLOPE = 1.13
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def half(dtype):
    return torch.finfo(dtype).eps / 2


def act(z, name):
    """Value and slope in 64 bits."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp_min(0), (z > 0).to(z)
    if name == "tanh":
        t = torch.tanh(z)
        return t, 1 - t * t
    if name == "gelu":
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return z * s, s + z * s * (1 - s)


def d(t):
    return None if t is None else t.detach().cpu().double()


def forward(x, w, bias=None, residual=None, name="none", gated=False, dtype=None):
    """(y, bound of y, pre, bound of pre) for the type of x; dtype: of y."""
    T = x.dtype
    dtype = dtype or T
    x, w, bias, residual = d(x), d(w), d(bias), d(residual)
    K = x.shape[-1]
    z = torch.matmul(x, w.mT)
    s = torch.matmul(x.abs(), w.abs().mT)
    if bias is not None:
        z = z + bias.unsqueeze(-2)
        s = s + bias.unsqueeze(-2).abs()
    ez = (K + 4) * U * s
    pre, epre = z, ez + half(T) * z.abs() * (1 + 1e-3) + TINY[T]
    if gated:
        f = z.shape[-1] // 2
        a, _ = act(z[..., :f], name)
        ea = SLOPE * ez[..., :f] + 16 * U * (z[..., :f].abs() + 1)
        y = a * z[..., f:]
        e = ea * z[..., f:].abs() + a.abs() * ez[..., f:] + ea * ez[..., f:] + U * y.abs()
    else:
        y, _ = act(z, name)
        e = SLOPE * ez + (0 if name == "none" else 16 * U * (z.abs() + 1))
        if residual is not None:
            y = y + residual
            e = e + U * y.abs()
    return y, e + half(dtype) * (y.abs() + e) + TINY[dtype], pre, epre


def backward(dy, x, w, pre, name="none", gated=False):
    """((dx, bound), (dw, bound), (db, bound)); operands without members receive sums over them."""
    T = dy.dtype
    h, tiny = half(T), TINY[T]
    members = next((t.shape[0] for t in (dy, x, w) if t.dim() == 3), None)
    dy64, x64, w64, pre = d(dy), d(x), d(w), d(pre)
    if gated:
        f = dy.shape[-1]
        a, s = act(pre[..., :f], name)
        u = pre[..., f:]
        dz = torch.cat((dy64 * u * s, dy64 * a), -1)
        e = torch.cat((dy64.abs() * u.abs() * 48 * U + 4 * U * (dy64 * u * s).abs(),
                       dy64.abs() * 16 * U * (pre[..., :f].abs() + 1) + 4 * U * (dy64 * a).abs()), -1)
        rounded = True
    else:
        s = 1.0 if name == "none" else act(pre, name)[1]
        dz = dy64 * s
        e = 0 * dz if name == "none" else dy64.abs() * 48 * U + 4 * U * dz.abs()
        rounded = name != "none"
    eb = e + 0.0
    if rounded:
        e = e + h * dz.abs() + tiny

    def total(t, shared):
        return t.sum(0) if shared and members is not None else t

    wide, rows = dz.shape[-1], dz.shape[-2]
    n = members or 1
    out = []
    # dx
    v = total(torch.matmul(dz, w64), x.dim() == 2)
    terms = wide * (n if x.dim() == 2 else 1)
    b = total(torch.matmul(e, w64.abs()) + (terms + 4) * U * torch.matmul(dz.abs(), w64.abs()), x.dim() == 2)
    out.append((v, b + h * v.abs() * (1 + 1e-3) + tiny))
    # dw
    v = total(torch.matmul(dz.mT, x64.expand(*dz.shape[:-1], x64.shape[-1])), w.dim() == 2)
    terms = rows * (n if w.dim() == 2 else 1)
    b = total(torch.matmul(e.mT, x64.abs().expand(*dz.shape[:-1], x64.shape[-1])) +
              (terms + 4) * U * torch.matmul(dz.abs().mT, x64.abs().expand(*dz.shape[:-1], x64.shape[-1])), w.dim() == 2)
    out.append((v, b + h * v.abs() * (1 + 1e-3) + tiny))
    # db
    v = total(dz.sum(-2), w.dim() == 2)
    b = total((eb + 68 * U * dz.abs()).sum(-2), w.dim() == 2)
    out.append((v, b + h * v.abs() * (1 + 1e-3) + U * v.abs() + tiny))
    return out


def check(name, got, want, bound):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    if got.numel() == 0:
        return
    assert torch.equal(torch.isnan(got), torch.isnan(want)), name
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), name
    err, b = (got - want)[fine].abs(), bound[fine]
    worst = (err / b.clamp_min(1e-300)).max().item() if err.numel() else 0.0
    assert bool((err <= b).all()), f"{name}: error {worst:.3g} times its bound, {(err > b).sum().item()} of {err.numel()}"
