"""Launches hold fewer than 2^32 work-items: members beyond that go in several launches, one member's product, dz or bias
gradient beyond it is refused before anything is enqueued (CPU only: workspace queries, the pointers are never followed)."""
import pytest

from paper_2212_04180_amd import esmi
from test_operator_refusals import FAKE, _adamw, _backward, _forward, _query

G = 1 << 24  # workgroups of 256 threads: one too many


def _dense(members, rows, k, f, dtype=1, shared_w=False):
    return _forward(dtype=dtype, y_dtype=dtype, members=members, rows=rows, out=f, x_member=rows * k, x_row=k, w_member=0 if shared_w else f * k, w_row=k,
                    bias_p=0, residual_p=0, y_member=rows * f, y_row=f, pre_p=0, **{"in": k})


def _grads(members, rows, k, f, want, act=2):
    one = dict(dx_p=0, dw_p=0, db_p=0)
    one[want + "_p"] = FAKE
    return _backward(members=members, rows=rows, out=f, act=act, dy_member=rows * f, dy_row=f, x_member=rows * k, x_row=k, w_member=f * k,
                     w_row=k, pre_member=rows * f, pre_row=f, dx_member=rows * k, dx_row=k, dw_member=f * k, dw_row=k, db_member=f,
                     **one, **{"in": k})


def _unsupported(name, packed):
    rc, _, msg = _query(name, packed)
    assert rc == esmi.ES_ERR_UNSUPPORTED and "launch holds" in msg, (rc, msg)
    # the call itself says so before it looks at its workspace
    assert getattr(esmi.lib(), name)(packed, None, 0, None) == esmi.ES_ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_members_are_never_too_many(dtype):
    for members in (G - 1, G, G + 1, (1 << 31) - 1):
        for rows, k, f in ((1, 8, 64), (1, 8, 256), (40, 8, 8)):
            assert _query("es_dense", _dense(members, rows, k, f, dtype))[0] == esmi.ES_OK, (members, rows, k, f)
    for members in (G + 1, (1 << 31) - 1):
        for want in ("dx", "dw", "db"):
            assert _query("es_dense_backward", _grads(members, 1, 8, 8, want))[0] == esmi.ES_OK
            assert _query("es_dense_backward", _grads(members, 65, 1, 1, want))[0] == esmi.ES_OK


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_one_members_product(dtype):
    # four waves of 16 outputs each, then tiles of 128 rows
    assert _query("es_dense", _dense(1, 1, 1, (G - 1) * 64, dtype))[0] == esmi.ES_OK
    _unsupported("es_dense", _dense(1, 1, 1, (G - 1) * 64 + 1, dtype))
    _unsupported("es_dense", _dense(3, 1, 1, (G - 1) * 64 + 1, dtype))
    assert _query("es_dense", _dense(1, (G - 1) * 128, 1, 1, dtype))[0] == esmi.ES_OK
    _unsupported("es_dense", _dense(1, (G - 1) * 128 + 1, 1, 1, dtype))
    # one network on many members' rows: one product, or, beyond what a launch holds of it, one per member
    for members in (1 << 16, (1 << 17) - 1):
        assert _query("es_dense", _dense(members, 1 << 14, 1, 1, dtype, shared_w=True))[0] == esmi.ES_OK


def test_gradients():
    # dz: chunks of 64 rows
    assert _query("es_dense_backward", _grads(1, (G - 1) * 64, 1, 1, "dx"))[0] == esmi.ES_OK
    _unsupported("es_dense_backward", _grads(1, (G - 1) * 64 + 1, 1, 1, "dx"))
    _unsupported("es_dense_backward", _grads(1, (G - 1) * 64 + 1, 1, 1, "db", act=0))
    # without an activation no dz is made
    assert _query("es_dense_backward", _grads(1, (G - 1) * 64 + 1, 1, 1, "dx", act=0))[0] == esmi.ES_OK
    _unsupported("es_dense_backward", _grads(1, (G - 1) * 128 + 1, 1, 1, "dx", act=0))
    # the bias gradient's columns, 16 to a workgroup of 64 threads
    most = ((1 << 26) - 1) * 16
    assert _query("es_dense_backward", _grads(1, 65, 1, most, "db"))[0] == esmi.ES_OK
    _unsupported("es_dense_backward", _grads(1, 65, 1, most + 1, "db"))


def test_adamw():
    rc, msg = _adamw(n=(G - 1) * 4096 + 1)
    assert rc == esmi.ES_ERR_ARG and "n is out of range" in msg
