"""Gradients of 16-bit layers (marked gpu): dz rounded to the type is the one rounding between the operands and the
sums, the same bits on every call."""
import pytest
import torch

import layercheck as L

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _P():
    import paper_2212_04180_amd as P
    return P


def _dz(dy, pre, act, gated):
    """dz in 64 bits, and how far an fp32 evaluation may be from it (layercheck.backward's terms)."""
    dy, pre = L.d(dy), L.d(pre)
    if not gated:
        z = dy * L.act(pre, act)[1]
        return z, dy.abs() * 48 * L.U + 4 * L.U * z.abs()
    f = dy.shape[-1]
    a, s = L.act(pre[..., :f], act)
    u = pre[..., f:]
    z = torch.cat((dy * u * s, dy * a), -1)
    return z, torch.cat((dy.abs() * u.abs() * 48 * L.U, dy.abs() * 16 * L.U * (pre[..., :f].abs() + 1)), -1) + 4 * L.U * z.abs()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,k,f,act,gated", [(512, 256, 512, "gelu", False), (250, 131, 253, "tanh", False), (12, 445, 980, "silu", False),
                                                (512, 256, 256, "silu", True), (100, 77, 129, "gelu", True)])
def test_dz_is_rounded_once(dtype, rows, k, f, act, gated):
    """Rounding keeps the order of numbers, so the kernel's dz lies between the roundings of dz64 - e and dz64 + e: for
    nearly all elements these are one number, and what is left is the sums' order ((K + 4) u sum|a||b|) and the result's
    own half step."""
    P = _P()
    g = torch.Generator(device="cuda").manual_seed(rows + k + f)
    wide = 2 * f if gated else f
    x = torch.randn(rows, k, generator=g, device="cuda").to(dtype)
    w = (torch.randn(wide, k, generator=g, device="cuda") * k ** -0.5).to(dtype)
    dy = (torch.randn(rows, f, generator=g, device="cuda") * 0.05).to(dtype)
    pre = torch.matmul(x.float(), w.float().mT).to(dtype)
    call = (lambda: P.gated_backward(dy, x, w, pre, act=act)) if gated else (lambda: P.dense_backward(dy, x, w, pre, act=act))
    dx, dw, _ = call()
    z, e = _dz(dy, pre, act, gated)
    lo, hi = (z - e).to(dtype).double(), (z + e).to(dtype).double()
    assert (lo == hi).double().mean() > 0.9  # the bounds below are close ones
    x64, w64 = L.d(x), L.d(w)
    for name, got, v, move, size, terms in (
            ("dx", dx, lo @ w64, (hi - lo) @ w64.abs(), lo.abs() @ w64.abs(), wide),
            ("dw", dw, lo.mT @ x64, (hi - lo).mT @ x64.abs(), lo.abs().mT @ x64.abs(), rows)):
        b = move + (terms + 4) * L.U * (size + move)
        L.check(name, got, v, b + L.half(dtype) * (v.abs() + b) + L.TINY[dtype])
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(call()[:2], (dx, dw)))


def test_dz_beyond_the_range_of_fp16():
    """A dz of 90,000 is infinite, and what it touches is not finite; one of 1e-9 is 0; the others stay as they are."""
    P = _P()
    x = torch.ones(3, 4, device="cuda", dtype=HF)
    w = torch.full((4, 4), 0.001, device="cuda", dtype=HF)
    pre = torch.tensor([[1.0, 1.0, 300.0, 1.0], [1.0, 1.0, 1e-5, 1e-5], [1.0, 1.0, 2.0, 2.0]], device="cuda").to(HF)
    dy = torch.tensor([[300.0, 1.0], [1e-4, 1e-4], [1.0, 1.0]], device="cuda").to(HF)
    dx, dw, _ = P.gated_backward(dy, x, w, pre, act="relu")
    assert bool(torch.isinf(dx[0]).all()) and bool(torch.isfinite(dx[1:]).all())
    assert bool(torch.isinf(dw[0]).all()) and bool(torch.isfinite(dw[1:]).all())
    # row 1: dg = 1e-4 * 1e-5 is below half of fp16's smallest, du = dy; row 2: dg = 2, du = 1
    want = 2 * float(dy[1, 0].item()) * float(w[0, 0].item())
    assert bool(((dx[1].double() - want).abs() <= 2.0 ** -25 + want * 2.0 ** -11).all())
    want = 6 * float(w[0, 0].item())
    assert bool(((dx[2].double() - want).abs() <= want * (2.0 ** -11 + 8 * L.U)).all())
