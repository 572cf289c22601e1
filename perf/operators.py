"""Cases that measure the operators of networks: what a user's program calls beside the evolution strategies.

  dense           y = act(x W^T + b) + residual, one network or one per member of a population
  dense_backward  its gradients dx, dW, db
  gated           h = act(x Wg^T + bg) * (x Wu^T + bu), W = [Wg; Wu]: the first half of a gated feed-forward block
  gated_backward  its gradients
  adamw           an AdamW step over many tensors, states in 32 bits or in 8 (e4m3, one scale per 256 elements;
                  the second moment is held as its square root)

A population's weights are views into the asked members [members][parameters], as es.ask(materialize=True) gives them
(cast where the case's type has 16 bits).  run() computes the plain form in 32 bits from elementary torch operations
where `own` is false, and calls the library where it is true.  exact() repeats the definitions in 64 bits.

Sums over up to 11,264 terms and Adam's states lose nothing that matters in 32 bits.  The 8-bit states are codes:
their sums are formed from separately rounded products on every side, so that a state next to a border between two
codes rounds the same way.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
F8 = torch.float8_e4m3fn
BLOCK = 256          # elements that share a scale of the 8-bit states
F8_MAX, F8_MIN = 448.0, 2.0 ** -9  # largest e4m3 value, smallest above zero
MLP_TENSORS = "16384,256,65536,256,4096,16"  # the 64-256-256-16 network
# one layer of a large network: four square matrices, three of a gated block, norms and ragged biases
LAYER_TENSORS = ",".join(str(n) for n in [4096 * 4096] * 4 + [11264 * 4096] * 3 + [4096, 4096, 11263, 77])


def _matrix(op, rows, k, f, dtype, members=0, act="none", bias=True, residual=False, keep=False, shared_x=False, rest=0,
            name=None):
    c = {"op": op, "members": members, "rows": rows, "in": k, "out": f, "dtype": dtype, "act": act, "bias": bias,
         "residual": residual, "keep": keep, "shared_x": shared_x, "rest": rest}
    return dict(c, name=name) if name else c


def _adamw(sizes, bits, grad, copy, name=None):
    c = {"op": "adamw", "sizes": sizes, "bits": bits, "grad": grad, "copy": copy}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a control policy's first layer, one observation per member of a population of 256: latency
        _matrix("dense", 1, 64, 256, "f32", members=256, act="tanh", rest=69904, name="dense_policy_step"),
        # one token through a square projection with the residual's addition: one reading of the weights
        _matrix("dense", 1, 4096, 4096, "bf16", bias=False, residual=True, name="dense_token"),
        # a hidden layer of a population on a batch of inputs of its own
        _matrix("dense", 256, 256, 256, "bf16", members=256, act="tanh", name="dense_population"),
        # training batch through a wide layer, the pre-activation kept for its gradient
        _matrix("dense", 8192, 4096, 11264, "bf16", act="gelu", keep=True, name="dense_train"),
        # gradients of a square layer in training
        _matrix("dense_backward", 8192, 4096, 4096, "bf16", act="gelu", name="dense_backward_train"),
        # analytic gradients of a population in full precision, ragged sizes, all members on the same inputs
        _matrix("dense_backward", 250, 131, 253, "f32", members=96, act="tanh", shared_x=True,
                name="dense_backward_population"),
        # four sequences decoded at once through a gated block's projections
        _matrix("gated", 4, 4096, 11264, "bf16", act="silu", bias=False, name="gated_decode"),
        # the same block in training
        _matrix("gated", 4096, 4096, 11264, "bf16", act="silu", bias=False, keep=True, name="gated_train"),
        # gradients of a smaller gated block, fp16
        _matrix("gated_backward", 2048, 2048, 5632, "f16", act="silu", name="gated_backward_train"),
        # the step of the 64-256-256-16 network: latency
        _adamw(MLP_TENSORS, 32, "f32", False, name="adamw_mlp"),
        # one layer of a large network in mixed precision: 16-bit gradients, a 16-bit copy for the next forward
        _adamw(LAYER_TENSORS, 32, "bf16", True, name="adamw_layer"),
        # the same with states in 8 bits, gradients in 32
        _adamw(LAYER_TENSORS, 8, "f32", False, name="adamw_layer_8bit"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("dense", "dense", "dense_backward", "gated", "gated_backward", "adamw"))
    if op == "adamw":
        while True:
            sizes = [_log(rng, 1, 40_000_000) for _ in range(_log(rng, 1, 18))]
            if sum(sizes) <= 200_000_000:
                break
        return _adamw(",".join(map(str, sizes)), rng.choice((8, 32)), rng.choice(("f32", "bf16", "f16")),
                      rng.random() < 0.5)
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    act = rng.choice(("silu", "gelu")) if op.startswith("gated") else rng.choice(("none", "relu", "tanh", "gelu", "silu"))
    odd = (lambda n: n) if rng.random() < 0.5 else (lambda n: max(8, n // 8 * 8))  # half of them in whole vectors
    while True:
        members = _log(rng, 2, 2048) if rng.random() < 0.5 else 0
        if members:
            rows, k, f = _log(rng, 1, 512), odd(_log(rng, 8, 1024)), odd(_log(rng, 8, 1024))
        else:
            rows, k, f = _log(rng, 1, 8192), odd(_log(rng, 16, 11264)), odd(_log(rng, 16, 11264))
        c = _matrix(op, rows, k, f, dtype, members=members, act=act, bias=rng.random() < 0.7,
                    residual=op == "dense" and rng.random() < 0.4, keep=op in ("dense", "gated") and rng.random() < 0.5,
                    shared_x=bool(members) and rng.random() < 0.5, rest=rng.choice((0, 0, 77, 1024)) if members else 0)
        w = work(c)
        if 2e5 <= w["bytes"] <= 1e9 and w["flops"] <= (1.5e11 if dtype == "f32" else 7e11):
            return c


# ---- inputs ---------------------------------------------------------------------------------------------------
def _lead(c, shared=False):
    return [c["members"]] if c["members"] and not shared else []


def _weights(c, g, wide):
    """w [.., wide, in] and bias [.., wide]; a population's are views into its members' parameters."""
    T, K = TYPES[c["dtype"]], c["in"]
    if c["members"]:
        flat = torch.randn(c["members"], wide * K + wide + c["rest"], generator=g, device="cuda")
        flat[:, :wide * K] *= K ** -0.5
        flat[:, wide * K:] *= 0.1
        flat = flat.to(T)
        w, b = flat[:, :wide * K].unflatten(1, (wide, K)), flat[:, wide * K:wide * K + wide]
    else:
        w = (torch.randn(wide, K, generator=g, device="cuda") * K ** -0.5).to(T)
        b = (torch.randn(wide, generator=g, device="cuda") * 0.1).to(T)
    return w, b if c["bias"] else None


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if c["op"] == "adamw":
        return _prepare_adamw(c, g)
    T, gated = TYPES[c["dtype"]], c["op"].startswith("gated")
    wide = c["out"] * (2 if gated else 1)
    x = torch.randn(*_lead(c, c["shared_x"]), c["rows"], c["in"], generator=g, device="cuda").to(T)
    w, b = _weights(c, g, wide)
    s = {"case": c, "x": x, "w": w, "b": b}
    if c["op"].endswith("backward"):
        # what the forward kept, and a gradient of a mean loss
        z = _product(x.float(), w.float().mT)
        s["pre"] = (z if b is None else z + b.float().unsqueeze(-2)).to(T)
        s["dy"] = (torch.randn(*_lead(c), c["rows"], c["out"], generator=g, device="cuda") * 0.05).to(T)
    elif c["residual"]:
        s["residual"] = torch.randn(*_lead(c), c["rows"], c["out"], generator=g, device="cuda").to(T)
    return s


def _sizes(c):
    return [int(n) for n in c["sizes"].split(",")]


def _prepare_adamw(c, g):
    """One flat allocation per kind of tensor, each tensor a view that starts at a multiple of 256 elements."""
    sizes = _sizes(c)
    at = [0]
    for n in sizes:
        at.append(at[-1] + -(-n // BLOCK) * BLOCK)
    total = at[-1]

    def split(flat, unit=1):
        return [flat[a // unit:a // unit + -(-n // unit)] for a, n in zip(at, sizes)]

    p = torch.randn(total, generator=g, device="cuda") * 0.02
    grad = (torch.randn(total, generator=g, device="cuda") * 1e-3).to(TYPES[c["grad"]])
    m = torch.randn(total, generator=g, device="cuda") * 3e-4
    v = torch.rand(total, generator=g, device="cuda") * 1.5e-6 + 1e-9
    s = {"case": c, "p": split(p), "g": split(grad), "step": 100, "flat": {"p": p}, "copies": None,
         "decay": [0.1 if n > 20000 else 0.0 for n in sizes]}
    if c["bits"] == 8:
        (m, ms), (v, vs) = _to8(m.view(-1, BLOCK), False), _to8(v.sqrt_().view(-1, BLOCK), True)
        m, v = m.view(-1), v.view(-1)
        s["m_scale"], s["v_scale"] = split(ms, BLOCK), split(vs, BLOCK)
        s["flat"].update(m_scale=ms, v_scale=vs)
    s["m"], s["v"] = split(m), split(v)
    s["flat"].update(m=m, v=v)
    if c["copy"]:
        s["flat"]["copy"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
        s["copies"] = split(s["flat"]["copy"])
    return s


# ---- the plain form -------------------------------------------------------------------------------------------
def _product(a, b):
    """Batched product; operands that are alike for all members are shared."""
    return torch.matmul(a, b)


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.clamp_min(z, 0)
    if act == "tanh":
        return torch.tanh(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z * torch.sigmoid(z)


def _act_grad(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "tanh":
        return 1 - torch.tanh(z).square()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


def _forward(s, W, gated):
    """y and z in the type W."""
    c = s["case"]
    z = _product(s["x"].to(W), s["w"].to(W).mT)
    if s["b"] is not None:
        z = z + s["b"].to(W).unsqueeze(-2)
    if gated:
        a, u = z.chunk(2, -1)
        y = _act(a, c["act"]) * u
    else:
        y = _act(z, c["act"])
        if "residual" in s:
            y = y + s["residual"].to(W)
    return y, z


def _backward(s, W, gated):
    """dx, dw and db in the type W."""
    c = s["case"]
    dy, z, x, w = s["dy"].to(W), s["pre"].to(W), s["x"].to(W), s["w"].to(W)
    if gated:
        a, u = z.chunk(2, -1)
        dz = torch.cat((dy * u * _act_grad(a, c["act"]), dy * _act(a, c["act"])), -1)
    else:
        dz = dy * _act_grad(z, c["act"])
    dw = _product(dz.mT, x)
    if c["members"] and c["shared_x"]:  # all members' contributions: one product over members and outputs
        dx = _product(dz.transpose(0, 1).flatten(1), w.flatten(0, 1))
    else:
        dx = _product(dz, w)
    return dx, dw, dz.sum(-2)


def _to8(t, root):
    """Codes and scales of blocks [.., 256]: nearest e4m3 of t / scale; the largest magnitude takes 448."""
    scale = (t.abs().amax(-1) * (1 / F8_MAX)).clamp_min(2.0 ** -126)
    q = t / scale.unsqueeze(-1)
    if root:  # a square root above zero stays above zero
        q = torch.where(t > 0, q.clamp_min(F8_MIN), q)
    return q.to(F8), scale


def _f32(v):
    """v rounded to fp32, as a Python float."""
    return torch.tensor(v, dtype=torch.float32).item()


def _constants(step, lr, beta1=0.9, beta2=0.999):
    b1, b2 = _f32(beta1), _f32(beta2)
    return b1, _f32(1 - b1), b2, _f32(1 - b2), _f32(1 - b1 ** step), _f32(1 - b2 ** step), _f32(lr), _f32(1e-8)


LR = 1e-3


def _adamw_plain(s):
    b1, o1, b2, o2, c1, c2, lr, eps = _constants(s["step"], LR)
    g = [t.float() for t in s["g"]]
    m, v = s["m"], s["v"]
    if s["case"]["bits"] == 8:
        parts = [_adamw8_plain(*a, b1, o1, b2, o2) for a in zip(g, m, v, s["m_scale"], s["v_scale"])]
        m, v = [a for a, _ in parts], [a for _, a in parts]
    else:
        torch._foreach_mul_(m, b1)
        torch._foreach_add_(m, g, alpha=o1)
        torch._foreach_mul_(v, b2)
        torch._foreach_addcmul_(v, g, g, value=o2)
    den = torch._foreach_div(v, c2)
    torch._foreach_sqrt_(den)
    torch._foreach_add_(den, eps)
    q = torch._foreach_div(m, c1)
    torch._foreach_div_(q, den)
    torch._foreach_mul_(s["p"], [1 - lr * d for d in s["decay"]])
    torch._foreach_add_(s["p"], q, alpha=-lr)
    if s["copies"] is not None:
        torch._foreach_copy_(s["copies"], s["p"])


def _adamw8_plain(g, m, v, ms, vs, b1, o1, b2, o2):
    """The moments after the step in 32 bits; the states receive their codes."""
    pad = -g.numel() % BLOCK

    def blocks(t):
        return torch.nn.functional.pad(t, (0, pad)).view(-1, BLOCK)

    gb = blocks(g)
    r = blocks(v.float()) * vs.unsqueeze(-1)
    m1 = blocks(m.float()) * ms.unsqueeze(-1) * b1 + gb * o1
    v1 = r * r * b2 + gb * gb * o2
    for state, scale, value in ((m, ms, m1), (v, vs, v1.sqrt())):
        code, sc = _to8(value, state is v)
        state.copy_(code.view(-1)[:g.numel()])
        scale.copy_(sc)
    return m1.view(-1)[:g.numel()], v1.view(-1)[:g.numel()]


# ---- one pass -------------------------------------------------------------------------------------------------
def run(state):
    s = state
    c = s["case"]
    op = c["op"]
    if op == "adamw":
        s["step"] += 1
        if own:
            import paper_2212_04180_amd as P
            P.adamw(s["p"], s["g"], s["m"], s["v"], s["step"], lr=LR, weight_decay=s["decay"],
                    m_scale=s.get("m_scale"), v_scale=s.get("v_scale"), copies=s["copies"])
        else:
            _adamw_plain(s)
        return dict(s["flat"])
    T, gated = TYPES[c["dtype"]], op.startswith("gated")
    if op.endswith("backward"):
        needs = (True, True, c["bias"])
        if own:
            import paper_2212_04180_amd as P
            f = P.gated_backward if gated else P.dense_backward
            dx, dw, db = f(s["dy"], s["x"], s["w"], pre=s["pre"], act=c["act"], needs=needs)
        else:
            dx, dw, db = (t.to(T) for t in _backward(s, torch.float32, gated))
        return {"dx": dx, "dw": dw, "db": db} if c["bias"] else {"dx": dx, "dw": dw}
    if own:
        import paper_2212_04180_amd as P
        if gated:
            r = P.gated(s["x"], s["w"], s["b"], act=c["act"], keep_pre=c["keep"])
        else:
            r = P.dense(s["x"], s["w"], s["b"], s.get("residual"), act=c["act"], keep_pre=c["keep"])
        return {"y": r[0], "pre": r[1]} if c["keep"] else {"y": r}
    y, z = _forward(s, torch.float32, gated)
    return {"y": y.to(T), "pre": z.to(T)} if c["keep"] else {"y": y.to(T)}


def work(case):
    c = case
    if c["op"] == "adamw":
        n = sum(_sizes(c))
        states = 16 if c["bits"] == 32 else 4 + 16 / BLOCK  # both moments, in and out, and their scales
        return {"bytes": n * (8 + SIZE[c["grad"]] + states + (2 if c["copy"] else 0)), "flops": 16 * n}
    M, B, K, F = max(1, c["members"]), c["rows"], c["in"], c["out"]
    wide = F * (2 if c["op"].startswith("gated") else 1)
    x = (1 if c["shared_x"] else M) * B * K
    w, b = M * wide * K, M * wide if c["bias"] else 0
    product = 2 * M * B * K * wide
    if c["op"].endswith("backward"):  # dy, pre, x and w in; dx, dw and db out
        return {"bytes": SIZE[c["dtype"]] * (M * B * (F + wide) + 2 * x + 2 * w + b), "flops": 2 * product}
    y = M * B * (F * (2 if c["residual"] else 1) + (wide if c["keep"] else 0))
    return {"bytes": SIZE[c["dtype"]] * (x + w + b + y), "flops": product}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------
def _exact_act(z, act):
    """Value and derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), torch.where(z > 0, 1.0, 0.0).to(z)
    if act == "tanh":
        t = torch.tanh(z)
        return t, 1.0 / torch.cosh(z).square()
    if act == "gelu":
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = 1.0 / (1.0 + torch.exp(-z))
    return z * s, s + z * s * (1.0 - s)


def _exact_adamw(c, s):
    b1, o1, b2, o2, c1, c2, lr, eps = _constants(s["step"] + 1, LR)
    flat = {k: (t if t.dtype == F8 else t.double()) for k, t in s["flat"].items()}
    at = 0
    for i, n in enumerate(_sizes(c)):
        e = at + n
        g = s["g"][i].double()
        if c["bits"] == 8:
            per = torch.arange(n, device="cuda") // BLOCK
            m = s["m"][i].double() * s["m_scale"][i].double()[per]
            v = (s["v"][i].double() * s["v_scale"][i].double()[per]).square()
        else:
            m, v = s["m"][i].double(), s["v"][i].double()
        m = b1 * m + o1 * g
        v = b2 * v + o2 * g * g
        p = s["p"][i].double() * (1.0 - lr * s["decay"][i]) - lr * (m / c1) / ((v / c2).sqrt() + eps)
        flat["p"][at:e] = p
        if c["copy"]:
            flat["copy"][at:e] = p
        if c["bits"] == 8:
            a, k = at // BLOCK, -(-n // BLOCK)
            for name, t in (("m", m), ("v", v.sqrt())):
                scale = torch.zeros(k, dtype=torch.float64, device="cuda").scatter_reduce_(0, per, t.abs(), "amax") / F8_MAX
                scale = scale.clamp_min(2.0 ** -126)
                flat[name + "_scale"][a:a + k] = scale
                q = t / scale[per]
                if name == "v":
                    q = torch.where(t > 0, q.clamp_min(F8_MIN), q)
                flat[name][at:e] = q.to(F8)
        else:
            flat["m"][at:e], flat["v"][at:e] = m, v
        at += -(-n // BLOCK) * BLOCK
    return {k: t.double() for k, t in flat.items()}


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "adamw":
        return _exact_adamw(c, s)
    x, w = s["x"].double(), s["w"].double()
    gated, F = c["op"].startswith("gated"), c["out"]
    if c["op"].endswith("backward"):
        z, dy = s["pre"].double(), s["dy"].double()
        if gated:
            a, da = _exact_act(z[..., :F], c["act"])
            dz = torch.empty_like(z)
            dz[..., :F], dz[..., F:] = dy * z[..., F:] * da, dy * a
        else:
            dz = dy * _exact_act(z, c["act"])[1]
        dx = torch.matmul(dz, w)
        if c["members"] and c["shared_x"]:
            dx = dx.sum(0)
        out = {"dx": dx, "dw": torch.matmul(dz.transpose(-1, -2), x)}
        return dict(out, db=dz.sum(-2)) if c["bias"] else out
    z = torch.matmul(x, w.transpose(-1, -2))
    if c["bias"]:
        z += s["b"].double()[..., None, :]
    if gated:
        y = _exact_act(z[..., :F], c["act"])[0] * z[..., F:]
    else:
        y = _exact_act(z, c["act"])[0]
        if c["residual"]:
            y += s["residual"].double()
    return {"y": y, "pre": z} if c["keep"] else {"y": y}
