"""Activations of 16-bit layers and their slopes (marked gpu) at every value of the type up to 13: within the half step
of the result's own size, far from zero too."""
import math

import pytest
import torch

import layercheck as L

pytestmark = pytest.mark.gpu

U = L.U


def _P():
    import paper_2212_04180_amd as P
    return P


def _values(dtype):
    """Every value of the type between -13 and 13."""
    top = torch.tensor(13.0).to(dtype).view(torch.int16).item()
    z = torch.arange(0, top + 1, dtype=torch.int16).view(dtype)
    return torch.cat((-z.flip(0), z)).unsqueeze(1).cuda()


def _exact(z, act):
    """Value, slope, and the sum of its terms' sizes, in 64 bits."""
    if act == "tanh":
        d = 1 / torch.cosh(z) ** 2
        return torch.tanh(z), d, d
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * torch.sigmoid(-z)), s * (1 + z.abs() * torch.sigmoid(-z))
    phi, pdf = 0.5 * torch.special.erfc(-z / math.sqrt(2.0)), torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return z * phi, phi + z * pdf, phi + z.abs() * pdf


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ["gelu", "tanh", "silu"])
def test_every_value(dtype, act):
    """A product of one term with 1 hands z over as it is.  In fp32 the value is within r = (2 z^2 + 32) u of its own size
    (the roundings of the exponent z^2 / 2 and its factor, three of u each on up to 85, the polynomial's and the
    reciprocal's; of tanh and silu the exponents 2 z and z, two of u each, so (4 |z| + 32) u), the slope within r of its
    terms'; then the half step.  (silu's 1 - s takes away from 1 what is next to it: its terms' sizes with u more.)  Results below 1e-36 may be flushed."""
    P = _P()
    z = _values(dtype)
    one = torch.ones(1, 1, dtype=dtype, device="cuda")
    v, d, size = _exact(L.d(z), act)
    r = (2 * L.d(z) ** 2 + 32 if act == "gelu" else 4 * L.d(z).abs() + 32) * U
    y, pre = P.dense(z, one, act=act, keep_pre=True)
    assert torch.equal(pre, z)
    b = r * v.abs() + 1e-36
    L.check("value", y, v, b + L.half(dtype) * (v.abs() + b) + L.TINY[dtype])
    L.check("in 32 bits", P.dense(z, one, act=act, out_dtype=torch.float32), v, b + U * v.abs())
    # few rows, tiles of 64 and the large ones evaluate alike
    for rows in (z[:7], z[:512].reshape(512, 1)):
        assert torch.equal(P.dense(rows, one, act=act), y[:rows.shape[0]])
    dx = P.dense_backward(torch.ones_like(z), z, one, pre, act=act, needs=(True, False, False))[0]
    b = r * size + 1e-36
    if act == "silu":
        b = b + 2 * U * (v.abs() + d.abs())
    L.check("slope", dx, d, b + L.half(dtype) * (d.abs() + b) + L.TINY[dtype])
    # the gate of a gated layer, times 1
    h, pre = P.gated(z, torch.cat((one, 0 * one)), torch.tensor([0.0, 1.0], device="cuda").to(dtype), act=act, keep_pre=True)
    assert torch.equal(h, y)
    dg = P.gated_backward(torch.ones_like(z), z, torch.cat((one, 0 * one)), pre, act=act, needs=(True, False, False))[0]
    assert torch.equal(dg, dx)


def test_slope_of_tanh_in_32_bits():
    """4 e / (1 + e)^2: the exponent -2 |z| is exact, the exponential within 2 u, eight more roundings."""
    P = _P()
    z = torch.linspace(-41, 41, 40001, device="cuda").unsqueeze(1)
    one = torch.ones(1, 1, device="cuda")
    dx = P.dense_backward(torch.ones_like(z), z, one, z, act="tanh", needs=(True, False, False))[0]
    d = 1 / torch.cosh(L.d(z)) ** 2
    L.check("slope", dx, d, 16 * U * d)
