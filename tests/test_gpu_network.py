"""The operators together as a program uses them (marked gpu): a gated block trained by its gradients and AdamW, the
population's networks evaluated layer by layer like the built-in neuroevolution problem, and a mean warm-started by
gradient steps handed to the strategy."""
import numpy as np
import pytest
import torch

import layercheck as L
from inputs import to_oracle
from oracle import oracle as O

pytestmark = pytest.mark.gpu


def _P():
    import paper_2212_04180_amd as P
    return P


def test_gated_block_trained_for_some_steps():
    """y = x + w2 (silu(x wg) (x wu)) on a fixed batch, loss half the squared distance: five steps in fp32 against the
    same five in 64 bits.  Sums of at most 64 terms carry about 64 u each way; Adam divides the gradient by its own
    size, so that a relative error of it moves a step by that share of lr: gradients here are at least 1e-3 of their
    largest in all but few places, where the step's error is at most lr itself; those are counted."""
    P = _P()
    g = torch.Generator(device="cuda").manual_seed(2)
    B, D, F, lr = 48, 24, 32, 1e-3
    x = torch.randn(B, D, generator=g, device="cuda")
    target = torch.randn(B, D, generator=g, device="cuda")
    params = [torch.randn(2 * F, D, generator=g, device="cuda") * D ** -0.5, torch.zeros(2 * F, device="cuda"),
              torch.randn(D, F, generator=g, device="cuda") * F ** -0.5, torch.zeros(D, device="cuda")]
    ref = [L.d(p) for p in params]
    rm, rv = [torch.zeros_like(p) for p in ref], [torch.zeros_like(p) for p in ref]
    s = P.adamw_state(params)
    x64, t64 = L.d(x), L.d(target)
    first = None
    for step in range(1, 6):
        w1, b1, w2, b2 = params
        h, pre = P.gated(x, w1, b1, keep_pre=True)
        y = P.dense(h, w2, b2, residual=x)
        dy = y - target
        dh, dw2, db2 = P.dense_backward(dy, h, w2)
        _, dw1, db1 = P.gated_backward(dh, x, w1, pre, needs=(False, True, True))
        P.adamw(params, [dw1, db1, dw2, db2], s["m"], s["v"], step, lr=lr, weight_decay=[0.1, 0, 0.1, 0])

        r1, c1, r2, c2 = ref
        z = x64 @ r1.mT + c1
        a, sl = L.act(z[:, :F], "silu")
        u = z[:, F:]
        d = (a * u) @ r2.mT + c2 + x64 - t64
        e = d @ r2
        dz = torch.cat((e * u * sl, e * a), 1)
        grads = [dz.mT @ x64, dz.sum(0), d.mT @ (a * u), d.sum(0)]
        for i, (p, gr) in enumerate(zip(ref, grads)):
            rm[i] = 0.9 * rm[i] + 0.1 * gr
            rv[i] = 0.999 * rv[i] + 0.001 * gr * gr
            q = (rm[i] / (1 - 0.9 ** step)) / ((rv[i] / (1 - 0.999 ** step)).sqrt() + 1e-8)
            ref[i] = p * (1 - lr * (0.1 if i % 2 == 0 else 0)) - lr * q
        loss = 0.5 * (d * d).sum().item()
        first = first or loss
        assert abs(0.5 * (dy * dy).sum().item() - loss) < 1e-4 * first
    total = sum(p.numel() for p in params)
    off = 0
    for p, r in zip(params, ref):
        err = (L.d(p) - r).abs()
        assert err.max().item() <= 5 * 2 * lr  # whatever a gradient's sign
        off += int((err > 5 * lr * 1e-3).sum())
    assert off <= 0.01 * total


def test_mixed_precision_copy_feeds_the_next_layer():
    """fp32 parameters, bf16 copies as the layers' weights: the copies follow the parameters."""
    P = _P()
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randn(40, 72, generator=g, device="cuda") * 0.1
    wb = w.bfloat16()
    x = torch.randn(30, 72, generator=g, device="cuda").bfloat16()
    s = P.adamw_state([w], bits=8)
    for step in range(1, 4):
        y, pre = P.dense(x, wb, act="tanh", keep_pre=True)
        dw = P.dense_backward(y, x, wb, pre, act="tanh", needs=(False, True, False))[1]
        P.adamw([w], [dw], s["m"], s["v"], step, lr=0.01, m_scale=s["m_scale"], v_scale=s["v_scale"], copies=[wb])
        assert torch.equal(wb, w.bfloat16())
        v, e, _, _ = L.forward(x, wb, None, None, "tanh")
        L.check("y", P.dense(x, wb, act="tanh"), v, e)


def test_population_layers_are_the_neuroevolution_problem():
    """The asked members' 64-256-256-16 networks, layer by layer through dense, score like es_eval: the same bf16
    operands, sums and activations to fp32's roundings, so that few hidden values round to another bf16 (the bar of
    the problem's own test with given weights, 1e-3)."""
    P = _P()
    cfg = P.ESConfig(num_dims=86544, popsize=16, num_runs=1, sigma=0.02, lr=0.01, seed=3, init=P.INIT_FANIN_NORMAL,
                     problem=P.PROB_MLP, maximize=1, mlp_batch=256, mlp_bf16=1)
    es = P.ES(cfg)
    pop = es.ask(materialize=True)[0]
    fit = es.eval()[0].double().cpu().numpy()
    oc = to_oracle(cfg)
    teacher = es.problem_data().cpu().numpy()
    xs, yt = O.mlp_inputs(oc, 0), None
    x = torch.tensor(xs, device="cuda").reshape(256, 64)
    net = torch.tensor(teacher, device="cuda").double()

    def layers(flat):
        at, out = 0, []
        for k, f in ((64, 256), (256, 256), (256, 16)):
            out.append((flat[..., at:at + k * f].unflatten(-1, (f, k)), flat[..., at + k * f:at + k * f + f]))
            at += k * f + f
        return out

    h = x.double()
    for i, (w, b) in enumerate(layers(net)):
        h = h @ w.mT + b
        if i < 2:
            h = torch.tanh(h)
    yt = h
    half = pop.bfloat16()
    h = x.bfloat16()
    for i, ((w, _), (_, b)) in enumerate(zip(layers(half), layers(pop))):
        # the problem keeps its biases in fp32: the product first, in fp32, then what a program adds
        z = P.dense(h, w, out_dtype=torch.float32)
        assert z.shape == (16, 256, w.shape[1])
        z = z + b.unsqueeze(1)
        h = torch.tanh(z).bfloat16() if i < 2 else z
    mse = ((h.double() - yt) ** 2).mean((1, 2)).cpu().numpy()
    assert np.all(np.abs(-mse - fit) <= 1e-3 * np.abs(fit)), (mse, fit)


def test_warm_start_of_the_mean():
    """Gradient steps on the mean's network, then the strategy goes on from there: its asked members are around it."""
    P = _P()
    cfg = P.ESConfig(num_dims=24 * 8 + 8, popsize=32, sigma=0.01, lr=0.01, seed=4, problem=P.PROB_NONE)
    es = P.ES(cfg)
    st = es.get_state()
    flat = st["m"][0].clone()
    w, b = flat[:192].view(8, 24), flat[192:]
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(64, 24, generator=g, device="cuda")
    m, v = st["m1"][0].clone(), st["v"][0].clone()
    parts = lambda t: [t[:192].view(8, 24), t[192:]]  # noqa: E731
    for step in range(1, 4):
        y, pre = P.dense(x, w, b, act="tanh", keep_pre=True)
        _, dw, db = P.dense_backward(y, x, w, pre, act="tanh", needs=(False, True, True))
        P.adamw([w, b], [dw, db], parts(m), parts(v), step, lr=0.01)
    es.set_state(flat[None], m[None], v[None], 3)
    pop = es.ask(materialize=True)[0]
    # antithetic pairs: their mean is the mean, to the members' roundings
    mid = (pop[:16].double() + pop[16:].double()) / 2
    assert (mid - flat.double()).abs().max().item() <= 2.0 ** -24 * pop.abs().max().item()
    h = P.dense(x.expand(32, -1, -1), pop[:, :192].view(32, 8, 24), pop[:, 192:], act="tanh")
    val, e, _, _ = L.forward(x, pop[:, :192].view(32, 8, 24), pop[:, 192:], None, "tanh")
    L.check("population", h, val, e)
