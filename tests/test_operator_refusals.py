"""What the operators of networks refuse, before any device call (CPU only: the
pointers here are never followed), and their workspace queries."""
import ctypes
import struct

import pytest
import torch

from paper_2212_04180_amd import esmi, operators

FWD = ["dtype", "y_dtype", "act", "reserved", "members", "rows", "in", "out",
       *[f"{m}_{f}" for m in ("x", "w", "bias", "residual", "y", "pre") for f in ("p", "member", "row")]]
BWD = ["dtype", "act", "members", "rows", "in", "out",
       *[f"{m}_{f}" for m in ("dy", "x", "w", "pre", "dx", "dw", "db") for f in ("p", "member", "row")]]
FAKE = 1 << 20  # an address that is aligned to everything


def _forward(gated=False, **kw):
    """A valid call of 3 members, 4 rows, 6 inputs and 8 outputs, but for kw."""
    wide = 16 if gated else 8
    a = dict(dtype=1, y_dtype=1, act=2, reserved=0, members=3, rows=4, out=8, x_p=FAKE, x_member=24, x_row=6, w_p=FAKE,
             w_member=6 * wide, w_row=6, bias_p=FAKE, bias_member=wide, bias_row=0, residual_p=0 if gated else FAKE,
             residual_member=32, residual_row=8, y_p=FAKE, y_member=32, y_row=8, pre_p=FAKE, pre_member=4 * wide, pre_row=wide)
    a["in"] = 6
    a.update(kw)
    return operators._FORWARD.pack(*(a[k] for k in FWD))


def _backward(gated=False, **kw):
    wide = 16 if gated else 8
    a = dict(dtype=1, act=2, members=3, rows=4, out=8, dy_p=FAKE, dy_member=32, dy_row=8, x_p=FAKE, x_member=24, x_row=6,
             w_p=FAKE, w_member=6 * wide, w_row=6, pre_p=FAKE, pre_member=4 * wide, pre_row=wide, dx_p=FAKE, dx_member=24,
             dx_row=6, dw_p=FAKE, dw_member=6 * wide, dw_row=6, db_p=FAKE, db_member=wide, db_row=0)
    a["in"] = 6
    a.update(kw)
    return operators._BACKWARD.pack(*(a[k] for k in BWD))


def _query(name, packed):
    n = ctypes.c_size_t(12345)
    rc = getattr(esmi.lib(), name + "_workspace")(packed, ctypes.byref(n))
    return rc, n.value, esmi.lib().es_last_error(None).decode()


def _refused(name, packed, word):
    rc, _, msg = _query(name, packed)
    assert rc == esmi.ES_ERR_ARG and word in msg and msg.startswith(name), (rc, msg)
    # the call itself says the same, without a workspace
    rc = getattr(esmi.lib(), name)(packed, None, 0, None)
    assert rc == esmi.ES_ERR_ARG and word in esmi.lib().es_last_error(None).decode()


def test_structs_have_the_headers_sizes():
    assert operators._FORWARD.size == 16 + 32 + 6 * 24
    assert operators._BACKWARD.size == 8 + 32 + 7 * 24
    assert struct.calcsize("=" + operators._TENSOR) == 72 and operators._ADAMW.size == 40


@pytest.mark.parametrize("name,gated", [("es_dense", False), ("es_gated", True)])
def test_forward(name, gated):
    assert _query(name, _forward(gated))[0] == esmi.ES_OK
    for kw, word in ((dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(y_dtype=2), "y_dtype"), (dict(act=5), "act"),
                     (dict(act=-1), "act"), (dict(reserved=1), "reserved"), (dict(rows=-1), "negative"),
                     (dict(members=-2), "negative"), (dict(rows=1 << 31), "2^31"), (dict(members=1 << 31), "2^31"),
                     (dict(x_p=0), "x is missing"), (dict(w_p=0), "w is missing"), (dict(y_p=0), "y is missing"),
                     (dict(x_p=FAKE + 1), "x is not aligned"), (dict(bias_p=FAKE + 1), "bias is not aligned"),
                     (dict(y_p=FAKE + 2, y_dtype=0), "y is not aligned"), (dict(x_row=-6), "x has a negative stride"),
                     (dict(w_member=-1), "w has a negative"), (dict(y_row=7), "y has rows that overlap"),
                     (dict(y_member=0), "y has members that overlap"), (dict(y_member=31), "y has members that overlap"),
                     (dict(pre_row=3), "pre has rows that overlap"), (dict(x_member=1 << 60), "x reaches beyond")):
        _refused(name, _forward(gated, **kw), word)
    # members interleaved within the rows are fine
    assert _query(name, _forward(gated, y_member=8, y_row=24))[0] == esmi.ES_OK
    _refused(name, _forward(gated, y_member=8, y_row=23), "overlap")
    if gated:
        _refused(name, _forward(gated, residual_p=FAKE), "residual")
        _refused(name, _forward(gated, out=(1 << 30) + 5), "2^31")
    # nothing to do needs nothing
    for kw in (dict(rows=0), dict(members=0), dict(out=0)):
        empty = _forward(gated, x_p=0, w_p=0, bias_p=0, residual_p=0, y_p=0, pre_p=0, **kw)
        assert _query(name, empty)[:2] == (esmi.ES_OK, 0)
        assert getattr(esmi.lib(), name)(empty, None, 0, None) == esmi.ES_OK
    assert getattr(esmi.lib(), name)(None, None, 0, None) == esmi.ES_ERR_ARG
    assert getattr(esmi.lib(), name + "_workspace")(_forward(gated), None) == esmi.ES_ERR_ARG


@pytest.mark.parametrize("name,gated", [("es_dense_backward", False), ("es_gated_backward", True)])
def test_backward(name, gated):
    assert _query(name, _backward(gated))[0] == esmi.ES_OK
    for kw, word in ((dict(dtype=7), "dtype"), (dict(act=9), "act"), (dict(rows=-1), "negative"), (dict(dy_p=0), "dy is missing"),
                     (dict(pre_p=0), "pre is missing"), (dict(x_p=0), "x is missing"), (dict(w_p=0), "w is missing"),
                     (dict(dx_p=FAKE + 1), "dx is not aligned"), (dict(dx_row=5), "dx has rows"), (dict(dw_member=5), "dw has members"),
                     (dict(db_member=3), "db has members"), (dict(out=1 << 31), "2^31")):
        _refused(name, _backward(gated, **kw), word)
    # sums over the members, skipped gradients and what those do not need
    for kw in (dict(dx_member=0), dict(dw_member=0, db_member=0), dict(dx_p=0, w_p=0), dict(dw_p=0, x_p=0), dict(db_p=0)):
        assert _query(name, _backward(gated, **kw))[0] == esmi.ES_OK, kw
    if not gated:
        assert _query(name, _backward(act=0, pre_p=0))[0] == esmi.ES_OK


@pytest.mark.parametrize("packed,name", ids=["dense_backward", "gated_backward", "dense"], argvalues=[(_backward(), "es_dense_backward"), (_backward(True), "es_gated_backward"),
                                         (_forward(members=1, rows=40, y_row=64, residual_row=64, pre_row=64, out=64, x_row=60000,
                                                   w_row=60000, **{"in": 60000}), "es_dense")])
def test_workspace_must_fit(packed, name):
    rc, n, _ = _query(name, packed)
    assert rc == esmi.ES_OK and n > 0
    call = getattr(esmi.lib(), name)
    assert call(packed, ctypes.c_void_p(FAKE), n - 1, None) == esmi.ES_ERR_ARG
    assert b"too small" in esmi.lib().es_last_error(None)
    assert call(packed, ctypes.c_void_p(FAKE + 16), n, None) == esmi.ES_ERR_ARG
    assert b"not aligned" in esmi.lib().es_last_error(None)
    assert call(packed, None, n, None) == esmi.ES_ERR_ARG


def _adamw(count=1, g_dtype=0, bits=32, copy_dtype=1, step=1, b1=0.9, b2=0.999, eps=1e-8, reserved=0, **kw):
    t = dict(p=FAKE, g=FAKE, m=FAKE, v=FAKE, ms=FAKE, vs=FAKE, copy=0, n=10, lr=0.1, wd=0.0)
    t.update(kw)
    head = operators._ADAMW.pack(count, g_dtype, bits, copy_dtype, step, b1, b2, eps, reserved)
    table = struct.pack("=" + operators._TENSOR, *(t[k] for k in ("p", "g", "m", "v", "ms", "vs", "copy", "n", "lr", "wd")))
    rc = esmi.lib().es_adamw(head, table, None)
    return rc, esmi.lib().es_last_error(None).decode()


def test_adamw():
    nan, inf = float("nan"), float("inf")
    for kw, word in ((dict(count=-1), "count"), (dict(g_dtype=3), "g_dtype"), (dict(bits=16), "state_bits"), (dict(step=0), "step"),
                     (dict(b1=1.0), "betas"), (dict(b2=-0.1), "betas"), (dict(b1=nan), "betas"), (dict(eps=-1.0), "eps"),
                     (dict(eps=inf), "eps"), (dict(reserved=1), "reserved"), (dict(lr=nan), "lr"), (dict(lr=-1.0), "lr"),
                     (dict(wd=inf), "weight_decay"), (dict(n=-1), "n is out of range"), (dict(p=0), "null"), (dict(g=0), "null"),
                     (dict(m=0), "null"), (dict(v=0), "null"), (dict(p=FAKE + 2), "aligned"), (dict(g=FAKE + 2), "aligned"),
                     (dict(m=FAKE + 1), "aligned"), (dict(bits=8, ms=0), "m_scale"), (dict(bits=8, vs=FAKE + 2), "aligned"),
                     (dict(copy=FAKE, copy_dtype=0), "copy_dtype"), (dict(copy=FAKE + 1), "aligned")):
        rc, msg = _adamw(**kw)
        assert rc == esmi.ES_ERR_ARG and word in msg and msg.startswith("es_adamw"), (kw, msg)
    assert _adamw(count=0)[0] == esmi.ES_OK
    assert _adamw(n=0, p=0, g=0, m=0, v=0)[0] == esmi.ES_OK
    assert esmi.lib().es_adamw(None, None, None) == esmi.ES_ERR_ARG


def test_binding_refuses_host_tensors_and_odd_shapes():
    x, w = torch.zeros(2, 3), torch.zeros(4, 3)
    with pytest.raises(ValueError, match="device"):
        operators.dense(x, w)
    with pytest.raises(ValueError, match="device"):
        operators.dense_backward(torch.zeros(2, 4), x, w)
    with pytest.raises(ValueError, match="device"):
        operators.adamw([x], [x], [x], [x], 1, lr=0.1)
    with pytest.raises(ValueError, match="32 or 8"):
        operators.adamw_state([x], bits=16)
    with pytest.raises(ValueError, match="activation"):
        operators._act("swish")


@pytest.mark.gpu
def test_binding_refusals_on_the_device():
    """Shapes, types, strides and members that do not go together."""
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)  # noqa: E731
    D, B = operators.dense, operators.dense_backward
    bf = torch.bfloat16
    for call, word in (
            (lambda: D(z(2, 3), z(4, 5)), "w is"), (lambda: D(z(2, 3), z(4, 3, dtype=bf)), "w is torch.bfloat16"),
            (lambda: D(z(2, 3, dtype=torch.int32), z(4, 3)), "fp32, bf16 or fp16"), (lambda: D(z(3), z(4, 3)), "dimensions"),
            (lambda: D(z(2, 3), z(4, 3).cpu()), "w is on cpu"), (lambda: D(z(3, 2).t(), z(4, 3)), "follow each other"),
            (lambda: D(z(2, 2, 3), z(5, 4, 3)), "members"), (lambda: D(z(2, 3), z(4, 3), z(5)), "bias has 5"),
            (lambda: D(z(2, 3), z(6, 4, 3), z(4)), "exactly where w has"), (lambda: D(z(2, 3), z(4, 3), residual=z(2, 5)), "residual is"),
            (lambda: D(z(2, 3), z(4, 3), out=z(2, 4, dtype=bf)), "output"), (lambda: D(z(2, 3), z(4, 3), out_dtype=bf), "output"),
            (lambda: D(z(2, 3), z(6, 4, 3), out=z(2, 4)), "members"), (lambda: operators.gated(z(2, 3), z(5, 3)), "even"),
            (lambda: B(z(2, 4), z(2, 3), z(4, 3), act="tanh"), "pre is needed"), (lambda: B(z(2, 4), z(2, 3), z(6, 4, 3)), "dy has no members"),
            (lambda: B(z(2, 4), z(1, 3), z(4, 3)), "x is"), (lambda: operators.gated_backward(z(2, 4), z(2, 3), z(4, 3), z(2, 8)), "w is")):
        with pytest.raises(ValueError, match=word):
            call()
    with pytest.raises(operators.EsError, match="overlap"):
        D(z(2, 3), z(4, 3), out=z(4).expand(2, 4))
    A = operators.adamw
    p = z(10)
    for call, word in (
            (lambda: A([p], [], [p], [p], 1, lr=1), "gradients"), (lambda: A([p], [z(9)], [p], [p], 1, lr=1), "sizes"),
            (lambda: A([p], [p], [z(10, dtype=bf)], [p], 1, lr=1), "states"), (lambda: A([p], [p.int()], [p], [p], 1, lr=1), "gradients"),
            (lambda: A([p, p], [p, p], [p, p], [p, p], 1, lr=1), "twice"), (lambda: A([p], [p], [p], [p], 1, lr=[1, 2]), "lr"),
            (lambda: A([z(20)[::2]], [p], [p], [p], 1, lr=1), "contiguous"), (lambda: A([p], [p], [p], [p], 1, lr=1, copies=[z(10)]), "copies"),
            (lambda: A([p], [p], [z(10, dtype=torch.uint8).view(torch.float8_e4m3fn)] * 1, [z(10, dtype=torch.uint8).view(torch.float8_e4m3fn)],
                       1, lr=1), "m_scale")):
        with pytest.raises(ValueError, match=word):
            call()
    with pytest.raises(operators.EsError, match="step"):
        A([p], [z(10)], [z(10)], [z(10)], 0, lr=1)
