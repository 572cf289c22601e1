"""The operators on a stream of the caller's (marked gpu): it waits for the operands, whose memory stays theirs until the
kernels have passed."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BUSY = 200_000_000  # cycles that a stream is kept waiting: about 0.1 s


def _P():
    import paper_2212_04180_amd as P
    return P


def _calls(P, s):
    """name, operands made on the current stream, call on s, the same on the current stream."""
    g = torch.Generator(device="cuda").manual_seed(1)

    def r(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    x, w, r1, dy, dh, pre = r(40, 64), r(96, 64), r(40, 96), r(40, 96), r(40, 48), r(40, 96)

    def adamw(stream):
        def run(p, g, m, v):
            P.adamw([p], [g], [m], [v], 2, lr=0.1, stream=stream)
            return p, m, v
        return run

    return [("dense", (x, w, r1), lambda x, w, r: P.dense(x, w, residual=r, act="tanh", stream=s),
             lambda x, w, r: P.dense(x, w, residual=r, act="tanh")),
            ("dense_backward", (dy, x, w, pre), lambda *a: P.dense_backward(*a, act="tanh", stream=s), lambda *a: P.dense_backward(*a, act="tanh")),
            ("gated", (x, w), lambda x, w: P.gated(x, w, stream=s), lambda x, w: P.gated(x, w)),
            ("gated_backward", (dh, x, w, pre), lambda *a: P.gated_backward(*a, stream=s), lambda *a: P.gated_backward(*a)),
            ("adamw", (x, r(40, 64), r(40, 64), r(40, 64).square()), adamw(s), adamw(None))]


def _all(out):
    return list(out) if isinstance(out, tuple) else [out]


def test_waits_for_operands_still_being_made():
    P = _P()
    s = torch.cuda.Stream()
    for name, operands, there, here in _calls(P, s):
        want = [t.clone() for t in _all(here(*(t * 2 for t in operands)))]
        torch.cuda.synchronize()
        torch.cuda._sleep(BUSY)
        got = _all(there(*(t * 2 for t in operands)))  # made behind the sleep
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name


def test_operands_freed_on_return_are_not_handed_out():
    P = _P()
    s = torch.cuda.Stream()
    for name, operands, there, here in _calls(P, s):
        want = [t.clone() for t in _all(here(*(t * 2 for t in operands)))]
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(BUSY)
        temporaries = [t * 2 for t in operands]
        held = {t.data_ptr() for t in temporaries}
        got = _all(there(*temporaries))
        written = {t.data_ptr() for t in got}
        del temporaries
        # what the caller's stream allocates next, and writes at once
        fresh = [torch.full_like(t, float("nan")) for t in operands]
        assert not s.query(), name  # still asleep: the kernels have not run
        assert not {t.data_ptr() for t in fresh} & (held - written), name
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
        del fresh, got


def test_the_current_stream_itself():
    P = _P()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for name, operands, there, here in _calls(P, s):
            a = [t.clone() for t in _all(there(*(t * 2 for t in operands)))]
            b = _all(here(*(t * 2 for t in operands)))
            assert all(torch.equal(p, q) for p, q in zip(a, b)), name
    torch.cuda.current_stream().wait_stream(s)


def test_captured_on_a_side_stream():
    """Within a capture the side stream joins it, as a stream that waits does; joined again it replays like the call."""
    P = _P()
    s = torch.cuda.Stream()
    for name, operands, there, here in _calls(P, s)[:4]:
        static = [t.clone() for t in operands]
        there(*static)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = _all(there(*static))
            torch.cuda.current_stream().wait_stream(s)
        for turn in range(4):
            for t in static:
                t.mul_(-1.125)
            graph.replay()
            want = _all(here(*static))
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (name, turn)
