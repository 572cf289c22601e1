"""What the operators do beside torch's autograd: it records none of them, so that operands which require a gradient are
refused where it would have to (CPU: the check; marked gpu: the calls)."""
import pytest
import torch

from paper_2212_04180_amd import operators


def test_the_check():
    t = torch.zeros(4, 3, requires_grad=True)
    for call in (lambda: operators._matrix("w", t, torch.float32, -1, None, None),
                 lambda: operators._vector("bias", t[0], torch.float32, -1, 3, None)):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad():
            call()
    operators._matrix("w", t.detach(), torch.float32, -1, None, None)


@pytest.mark.gpu
def test_operands_that_require_a_gradient():
    D, G, BD, BG = operators.dense, operators.gated, operators.dense_backward, operators.gated_backward

    def z(*s, **k):
        return torch.randn(*s, device="cuda", **k)

    plain = dict(x=z(2, 3), w=z(4, 3), bias=z(4), residual=z(2, 4), out=z(2, 4))
    for name in plain:
        args = {k: v.clone().requires_grad_(k == name) for k, v in plain.items()}
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            D(**args)
        with torch.no_grad():
            y = D(**args)
        assert not y.requires_grad or name == "out"
        if name != "out":
            assert torch.equal(y, D(**{k: v.detach() for k, v in plain.items()}))
    leaf = z(4, 3, requires_grad=True)
    for call, name in ((lambda: G(plain["x"], leaf), "w"), (lambda: BD(plain["residual"], plain["x"], leaf), "w"),
                       (lambda: BD(plain["residual"], plain["x"], plain["w"], leaf.new_zeros(2, 4).requires_grad_(), act="tanh"), "pre"),
                       (lambda: BG(z(2, 2, requires_grad=True), plain["x"], leaf.detach(), z(2, 4)), "dy")):
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            call()
        with torch.no_grad():
            call()


@pytest.mark.gpu
def test_within_a_function_of_the_users_own():
    """A torch.autograd.Function around a layer and its gradient: autograd calls both without recording."""

    class Dense(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, pre = operators.dense(x, w, b, act="tanh", keep_pre=True)
            ctx.save_for_backward(x, w, pre)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w, pre = ctx.saved_tensors
            return operators.dense_backward(dy.contiguous(), x, w, pre, act="tanh")

    g = torch.Generator(device="cuda").manual_seed(1)
    args = [torch.randn(*s, generator=g, device="cuda", requires_grad=True) for s in ((9, 24), (16, 24), (16,))]
    c = torch.randn(9, 16, generator=g, device="cuda")
    (Dense.apply(*args) * c).sum().backward()
    want = torch.autograd.grad((torch.tanh(args[0].double() @ args[1].double().mT + args[2].double()) * c).sum(), args)
    for a, w in zip(args, want):
        # sums of at most 24 terms of size 1, some ten roundings each way
        assert (a.grad - w).abs().max().item() <= 64 * 2.0 ** -24 * 24


@pytest.mark.gpu
def test_changed_tensors_are_known_as_changed():
    """Autograd refuses to go back through a tensor that it saved and an operator has overwritten since."""
    D = operators.dense
    x, w = torch.randn(5, 8, device="cuda"), torch.randn(6, 8, device="cuda")
    a = torch.randn(5, 6, device="cuda", requires_grad=True)
    saved = a.exp()  # its gradient is itself
    with torch.no_grad():
        D(x, w, out=saved)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        saved.sum().backward()
    saved = a.exp()
    with torch.no_grad():
        D(x, w, residual=saved, out=saved)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        saved.sum().backward()

    p = [torch.randn(n, device="cuda", requires_grad=True) for n in (300, 7)]
    for bits in (32, 8):
        s = operators.adamw_state(p, bits)
        g = [torch.randn_like(t) for t in p]
        copies = [torch.zeros(t.shape, device="cuda", dtype=torch.bfloat16) for t in p]
        before = {k: [t._version for t in ts] for k, ts in (("p", p), ("copies", copies), ("g", g), *s.items())}
        loss = (p[0] * p[0].detach().clone().requires_grad_()).sum()
        operators.adamw(p, g, s["m"], s["v"], 1, lr=0.1, m_scale=s.get("m_scale"), v_scale=s.get("v_scale"), copies=copies)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        for k, ts in (("p", p), ("copies", copies), *s.items()):
            assert all(t._version > v for t, v in zip(ts, before[k])), (bits, k)
        assert [t._version for t in g] == before["g"]
    with torch.inference_mode():  # tensors without a version
        q = [torch.randn(9, device="cuda")]
        s = operators.adamw_state(q)
        operators.adamw(q, [torch.ones(9, device="cuda")], s["m"], s["v"], 1, lr=0.1)
        D(x, w, out=torch.empty(5, 6, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_rows_of_one_tensor_as_the_lists(bits):
    """Lists may be a tensor's rows, as well for copies and scales; all of it counts as changed."""
    p, g = torch.zeros(3, 256, device="cuda"), torch.ones(3, 256, device="cuda")
    s = operators.adamw_state(list(p), bits)
    s = {k: torch.stack([t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in ts]) for k, ts in s.items()}
    if bits == 8:
        s["m"], s["v"] = (s[k].view(torch.float8_e4m3fn) for k in ("m", "v"))
    copies = torch.zeros(3, 256, device="cuda", dtype=torch.bfloat16)
    before = copies._version
    operators.adamw(p, g, s["m"], s["v"], 1, lr=0.5, m_scale=s.get("m_scale"), v_scale=s.get("v_scale"), copies=copies)
    assert bool(((p + 0.5).abs() < 1e-6).all()) and torch.equal(copies, p.bfloat16()) and copies._version > before
