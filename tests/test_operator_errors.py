"""Errors of the operators' calls: a failed call is not made a second time (CPU)."""
import types

import pytest

from paper_2212_04180_amd import esmi, operators


class _Library:
    """es_op that answers as told, one answer a call, and its workspace query."""

    def __init__(self, answers, need):
        self.answers, self.need, self.calls = list(answers), need, []

    def es_op(self, packed, workspace, n, stream):
        self.calls.append((workspace, n))
        return self.answers.pop(0)

    def es_op_workspace(self, packed, n):
        n._obj.value = self.need
        return esmi.ES_OK

    def es_last_error(self, handle):
        return b"es_op: what it was"


@pytest.fixture
def launch(monkeypatch):
    def run(answers, need):
        lib = _Library(answers, need)
        monkeypatch.setattr(operators.esmi, "lib", lambda: lib)
        monkeypatch.setattr(operators.torch.cuda, "current_device", lambda: 0)
        monkeypatch.setattr(operators, "_stream", lambda device: 7)
        monkeypatch.setattr(operators.torch, "empty", lambda n, **kw: types.SimpleNamespace(data_ptr=lambda: 4096))
        try:
            operators._launch("es_op", b"", 0)
        except operators.EsError as e:
            assert "what it was" in str(e)
            return lib.calls, e.args
        return lib.calls, None
    return run


def test_calls_and_their_workspace(launch):
    assert launch([esmi.ES_OK], 0) == ([(None, 0)], None)
    # refused without a workspace: asked for its size and called with one
    assert launch([esmi.ES_ERR_ARG, esmi.ES_OK], 512) == ([(None, 0), (4096, 512)], None)


@pytest.mark.parametrize("rc", [esmi.ES_ERR_HIP, esmi.ES_ERR_UNSUPPORTED])
@pytest.mark.parametrize("need", [0, 512])
def test_a_failed_call_is_not_repeated(launch, rc, need):
    """What it enqueued may have run: a residual written in place would be added twice."""
    calls, error = launch([rc, esmi.ES_OK], need)
    assert calls == [(None, 0)] and error is not None


def test_a_refused_call_without_a_workspace(launch):
    calls, error = launch([esmi.ES_ERR_ARG, esmi.ES_ERR_ARG], 0)
    assert error is not None and len(calls) <= 2  # refused calls have enqueued nothing
