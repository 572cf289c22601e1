"""Outputs that share memory with what a layer still reads: the binding's own check (CPU), and its refusals (marked gpu); streams
of another device."""
import random
from types import SimpleNamespace

import pytest
import torch

from paper_2212_04180_amd import operators


def _addresses(t):
    e = t.element_size()
    at = {t.data_ptr()} if t.numel() else set()
    for n, s in zip(t.shape, t.stride()):
        at = {a + i * s * e for a in at for i in range(n)}
    return {a + j for a in at for j in range(e)}


def test_overlap_is_never_missed():
    """Against every byte of random views, of two types, with and without members."""
    rng = random.Random(3)
    buf = torch.zeros(400)
    seen = [0, 0]
    for _ in range(3000):
        views = []
        for _ in range(2):
            base = buf if rng.random() < 0.7 else buf.view(torch.bfloat16)
            dims = rng.choice((2, 3))
            shape = [rng.randint(0 if rng.random() < 0.1 else 1, 4) for _ in range(dims)]
            stride = [rng.choice((0, 1, 3, 4, 8, 12, 16, 24, 48)) for _ in range(dims - 1)] + [1]
            views.append(base.as_strided(shape, stride, rng.randint(0, 60)))
        shared = bool(_addresses(views[0]) & _addresses(views[1]))
        for a, b in (views, views[::-1]):
            said = operators._overlap(a, b)
            assert said or not shared, (a.shape, a.stride(), b.shape, b.stride())
        seen[shared] += said == shared
    assert min(seen) > 300


def test_views_side_by_side_are_apart():
    o = operators._overlap
    buf = torch.zeros(6, 40)
    assert not o(buf[:, :16], buf[:, 16:40]) and not o(buf[:, 16:40], buf[:, :16])  # columns of one buffer
    assert not o(buf[:3], buf[3:]) and not o(buf[::2], buf[1::2])  # rows of it
    assert o(buf[:, :17], buf[:, 16:40]) and o(buf, buf) and o(buf[2:4], buf[3:5])
    arena = torch.zeros(5, 100)  # members' own inputs and outputs behind each other
    x, y = arena[:, 3:27].unflatten(1, (4, 6)), arena[:, 27:59].unflatten(1, (4, 8))
    assert not o(x, y) and not o(y, x) and o(x, arena[:, 26:58].unflatten(1, (4, 8)))
    rows = torch.zeros(4, 5, 14)  # members within the rows
    assert not o(rows[..., :6].transpose(0, 1), rows[..., 6:].transpose(0, 1))
    assert not o(torch.zeros(2, 3), torch.zeros(2, 3)) and not o(buf[:0], buf)


def test_a_stream_of_another_device_is_refused():
    """Without it the kernels would run on the operands' device, on whichever stream is current there."""
    stream = SimpleNamespace(device=torch.device("cuda", 1))
    here, there = (SimpleNamespace(is_cuda=True, device=torch.device("cuda", i)) for i in (0, 1))
    for tensors in ([here], [there, None, here]):
        with pytest.raises(ValueError, match="stream is on cuda:1, an operand on cuda:0"):
            operators._on(stream, tensors, lambda: pytest.fail("called"))


@pytest.mark.gpu
def test_out_within_the_operands_is_refused():
    D, G = operators.dense, operators.gated
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(40, 32, device="cuda").to(dtype)
        w = torch.randn(32, 32, device="cuda").to(dtype)
        b = torch.zeros(32, device="cuda", dtype=dtype)
        keep = x.clone(), w.clone()
        with pytest.raises(ValueError, match="shares memory with x"):
            D(x, w, out=x)
        with pytest.raises(ValueError, match="shares memory with w"):
            D(x[:32], w, out=w)
        with pytest.raises(ValueError, match="shares memory with bias"):
            D(x[:1], w, b, out=b.view(1, 32))
        with pytest.raises(ValueError, match="shares memory with x"):
            G(x, w, out=x[:, :16])
        buf = torch.zeros(41, 32, device="cuda", dtype=dtype)
        with pytest.raises(ValueError, match="not the residual itself"):
            D(x, w, residual=buf[:40], out=buf[1:])
        with pytest.raises(ValueError, match="not the residual itself"):
            D(x.expand(3, 40, 32), w, residual=buf[:40], out=buf[:40].expand(3, 40, 32))
        assert torch.equal(x, keep[0]) and torch.equal(w, keep[1]) and not bool(buf.any())
        # beside each other in one buffer, and the residual through another view of it
        wide = torch.zeros(40, 64, device="cuda", dtype=dtype)
        wide[:, :32] = x
        assert torch.equal(D(wide[:, :32], w, out=wide[:, 32:]), D(x, w)) and torch.equal(wide[:, :32], x)
        r = x.clone()
        want = D(x, w, residual=x)
        assert torch.equal(D(x, w, residual=r, out=r.view(40, 32)), want) and torch.equal(r, want)


def test_adamw_tensors_listed_twice():
    """Pointers as adamw gathers them: params, grads, m, v, scales, copies."""
    ok = [[10, 20], [30, 40], [50, 60], [70, 80], [0, 0], [0, 0], [0, 0]]
    operators._distinct(ok, [5, 6], 32, False)
    operators._distinct([*ok[:6], [90, 100]], [5, 6], 32, True)
    operators._distinct([*ok[:4], [110, 120], [130, 140], [90, 100]], [5, 6], 8, True)
    operators._distinct([ok[0], [30, 30], *ok[2:]], [5, 6], 32, False)  # one gradient for two is only read
    operators._distinct([[0, 20], [0, 40], [0, 60], [0, 80], *ok[4:]], [0, 6], 32, False)  # empty tensors
    operators._distinct([[20, 20], [20, 40], *ok[2:]], [0, 6], 32, False)
    for at, value in ((2, [50, 50]), (3, [50, 80]), (2, [10, 60]), (3, [70, 20])):
        cols = [*ok[:at], value, *ok[at + 1:]]
        with pytest.raises(ValueError, match="listed twice"):
            operators._distinct(cols, [5, 6], 32, False)
    for at, value in ((4, [110, 110]), (5, [130, 110]), (6, [90, 70]), (6, [10, 90])):
        cols = [*ok[:4], [110, 120], [130, 140], [90, 100]]
        cols[at] = value
        with pytest.raises(ValueError, match="listed twice"):
            operators._distinct(cols, [5, 6], 8, True)
    for grads in ([10, 40], [30, 60], [80, 40]):
        with pytest.raises(ValueError, match="a gradient is also"):
            operators._distinct([ok[0], grads, *ok[2:]], [5, 6], 32, False)


@pytest.mark.gpu
def test_adamw_refuses_shared_states():
    p, g, m, v = ([torch.ones(9, device="cuda") for _ in range(2)] for _ in range(4))
    for call, word in ((lambda: operators.adamw(p, g, [m[0], m[0]], v, 1, lr=0.1), "twice"), (lambda: operators.adamw(p, g, m, m, 1, lr=0.1), "twice"),
                       (lambda: operators.adamw(p, p, m, v, 1, lr=0.1), "gradient is also"), (lambda: operators.adamw([p[0], p[0]], g, m, v, 1, lr=0.1), "twice")):
        with pytest.raises(ValueError, match=word):
            call()
    assert all(bool((t == 1).all()) for ts in (p, g, m, v) for t in ts)
    operators.adamw(p, [g[0], g[0]], m, v, 1, lr=0.1)
    assert torch.equal(p[0], p[1])
