"""Dense and gated layers and their gradients (marked gpu) against plain forms
in 64 bits, within the bounds derived in layercheck.py: types, activations,
sizes from zero and one to several tiles, members, shared operands, strides,
alignments, NaN beside and within the data, streams and graphs."""
import pytest
import torch

import layercheck as L

pytestmark = pytest.mark.gpu

BF, HF, SF = torch.bfloat16, torch.float16, torch.float32
TYPES = [SF, BF, HF]


def _P():
    import paper_2212_04180_amd as P
    return P


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rand(g, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _case(seed, dtype, members, rows, k, f, act, gated=False, bias=True, residual=False, shared_x=False, shared_w=False):
    """Operands of a layer; members None: none."""
    g = _gen(seed)
    wide = 2 * f if gated else f
    lead = [] if members is None else [members]
    x = _rand(g, *([] if shared_x else lead), rows, k, dtype=dtype)
    w = _rand(g, *([] if shared_w else lead), wide, k, dtype=dtype, scale=max(1, k) ** -0.5)
    b = _rand(g, *([] if shared_w else lead), wide, dtype=dtype, scale=0.3) if bias else None
    r = _rand(g, *lead, rows, f, dtype=dtype) if residual else None
    dy = _rand(g, *lead, rows, f, dtype=dtype, scale=0.1)
    return x, w, b, r, dy


def _check(seed, dtype, members, rows, k, f, act, gated=False, **kw):
    """Forward with the pre-activation kept, then the gradients."""
    P = _P()
    print("layer", dtype, members, rows, k, f, act, "gated" if gated else "", kw, flush=True)
    x, w, b, r, dy = _case(seed, dtype, members, rows, k, f, act, gated, **kw)
    if gated:
        y, pre = P.gated(x, w, b, act=act, keep_pre=True)
        grads = P.gated_backward(dy, x, w, pre, act=act)
    else:
        y, pre = P.dense(x, w, b, r, act=act, keep_pre=True)
        grads = P.dense_backward(dy, x, w, pre, act=act)
    torch.cuda.synchronize()
    vy, by, vp, bp = L.forward(x, w, b, r, act, gated)
    L.check("y", y, vy, by)
    # all operands but the residual shared: the same pre for every member
    L.check("pre", pre, vp.expand(pre.shape), bp.expand(pre.shape))
    for name, got, (v, bound) in zip(("dx", "dw", "db"), grads, L.backward(dy, x, w, pre, act, gated)):
        L.check(name, got, v, bound)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["none", "relu", "tanh", "gelu", "silu"])
def test_activations(dtype, act):
    _check(1, dtype, None, 37, 70, 50, act, residual=True)
    _check(2, dtype, None, 19, 40, 33, act, gated=True)


SIZES = [  # rows, in, out: nothing, one, odd, about the tiles' edges, long sums
    (0, 5, 7), (5, 0, 7), (5, 7, 0), (1, 1, 1), (1, 64, 256), (2, 3, 5), (3, 1000, 1), (1, 1, 300), (16, 16, 16),
    (17, 33, 65), (64, 64, 64), (65, 127, 129), (127, 128, 255), (128, 256, 128), (129, 31, 257), (8, 4099, 24),
    (300, 72, 8), (4, 2048, 512), (1000, 24, 40), (257, 520, 264),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,k,f", SIZES)
def test_sizes(dtype, rows, k, f):
    _check(rows + k + f, dtype, None, rows, k, f, "tanh", residual=True)
    _check(rows + k + f, dtype, None, rows, k, f, "silu", gated=True, bias=rows % 2 == 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("members", [0, 1, 2, 7, 65])
@pytest.mark.parametrize("shared", [(False, False), (True, False), (False, True), (True, True)])
def test_members(dtype, members, shared):
    kw = dict(shared_x=shared[0], shared_w=shared[1])
    for rows, k, f in ((1, 24, 40), (9, 33, 17), (130, 64, 72)):
        _check(members, dtype, members, rows, k, f, "gelu", residual=True, **kw)
        _check(members, dtype, members, rows, k, f, "tanh", gated=True, **kw)


@pytest.mark.parametrize("dtype", TYPES)
def test_large(dtype):
    """Several tiles each way, whole 16-byte pieces and ragged."""
    for rows, k, f in ((512, 512, 768), (700, 640, 520), (509, 333, 771)):
        _check(3, dtype, None, rows, k, f, "gelu", residual=True)
        _check(4, dtype, None, rows, k, f, "silu", gated=True)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("members,rows,k,f", [
    (200, 64, 8, 64), (200, 72, 136, 264), (2, 2568, 200, 2632),  # ragged tiles, one step, odd and even numbers of steps
    (200, 264, 64, 72), (None, 4096, 128, 3088), (None, 3600, 192, 3856)])
def test_many_tiles(dtype, members, rows, k, f):
    """Products that fill the chip with tiles of the matrix cores' own kernels, whole 16-byte pieces; long ones' gradients
    by sums over the members."""
    _check(21, dtype, members, rows, k, f, "silu", residual=True)
    _check(22, dtype, members, rows, k, f // 2, "gelu", gated=True, bias=False)
    if members == 200:
        _check(23, dtype, members, rows, k, f, "relu", shared_x=True)
        _check(24, dtype, members, rows, k, f, "none", shared_w=True)


@pytest.mark.parametrize("dtype,rows,k,f", [(BF, 4104, 1096, 4096), (HF, 4360, 1024, 4088), (BF, 4104, 4096, 4104)])
def test_tiles_left_over(dtype, rows, k, f):
    """A few tiles behind full rounds of the chip's: their sums are made in parts."""
    _check(28, dtype, None, rows, k, f, "silu", residual=True)
    if k < 2000:
        _check(29, dtype, None, rows, k, f // 2, "gelu", gated=True)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_all_tiles_in_parts(dtype):
    """Long sums of too few tiles to fill the chip: every tile is made in parts, in the product and in its gradients."""
    _check(40, dtype, None, 1544, 10248, 1800, "gelu", residual=True)
    _check(41, dtype, None, 1544, 10248, 1032, "silu", gated=True)
    _check(42, dtype, None, 1800, 1544, 10248, "tanh")
    _check(43, dtype, None, 10248, 1544, 1800, "relu")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("members,rows,k,f", [(None, 128, 520, 49160), (None, 136, 64, 49160), (None, 49160, 200, 128),
                                              (200, 136, 136, 264), (200, 128, 72, 136)])
def test_thin_products(dtype, members, rows, k, f):
    """About as wide as one of the smaller tiles, and long."""
    _check(44, dtype, members, rows, k, f, "silu", residual=True)
    _check(45, dtype, members, rows, k, f // 2, "gelu", gated=True, bias=False)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("members,rows,k,f,kw", [
    (None, 4100, 1031, 2051, {}), (None, 2049, 2052, 2047, {}), (3, 2050, 1031, 1029, {}), (3, 1401, 1031, 2051, dict(shared_w=True)),
    (3, 1401, 1031, 2051, dict(shared_x=True))])
def test_large_and_ragged(dtype, members, rows, k, f, kw):
    """Sizes whose operands are copied into whole 16-byte pieces first, odd addresses among them."""
    _check(25, dtype, members, rows, k, f, "tanh", **kw)
    _check(26, dtype, members, rows, k, f // 2, "silu", gated=True, bias=False, **kw)


def test_large_and_ragged_without_activation():
    """dy itself is the operand: odd rows, a padded view with NaN in its gaps."""
    P = _P()
    x, w, b, _, dy = _case(27, BF, None, 2049, 2050, 2051, "none")
    big = torch.full((2049, 2060), float("nan"), dtype=BF, device="cuda")
    big[:, 3:2054] = dy
    for name, got, (v, bound) in zip(("dx", "dw", "db"), P.dense_backward(big[:, 3:2054], x, w), L.backward(dy, x, w, None)):
        L.check(name, got, v, bound)


def test_large_sums_over_members():
    """One network on many members, and one input for many networks: long reductions."""
    for dtype in TYPES:
        _check(5, dtype, 300, 8, 64, 48, "tanh", shared_w=True)
        _check(6, dtype, 300, 40, 24, 32, "tanh", shared_x=True)
        _check(7, dtype, None, 20000, 16, 24, "tanh")


def test_many_members():
    P = _P()
    x, w, b, _, _ = _case(8, BF, 70001, 1, 8, 8, "relu")
    y = P.dense(x, w, b, act="relu")
    v, e, _, _ = L.forward(x, w, b, None, "relu")
    L.check("y", y, v, e)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_alignment_and_what_lies_between(dtype):
    """Rows of views: odd offsets, odd pitches, NaN in every gap of the operands (read by mistake it would spread), and
    the gaps of the outputs left as they were."""
    P = _P()
    for off, pad in ((0, 8), (1, 0), (3, 5), (8, 13)):
        for members, rows, k, f, gated in ((None, 33, 45, 29, False), (3, 18, 64, 40, False), (3, 5, 37, 66, True),
                                           (None, 140, 136, 132, True), (2, 1, 129, 50, False)):
            print("strides", dtype, off, pad, members, rows, k, f, gated, flush=True)
            x, w, b, r, dy = _case(9, dtype, members, rows, k, f, "gelu", gated, residual=not gated)

            def spread(t):
                lead, (i, j) = t.shape[:-2], t.shape[-2:]
                big = torch.full((*lead, i + 2, j + off + pad), float("nan"), dtype=dtype, device="cuda")
                v = big[..., 1:1 + i, off:off + j]
                v.copy_(t)
                return v

            xs, ws, rs, ds = spread(x), spread(w), spread(r) if r is not None else None, spread(dy)
            lead = [] if members is None else [members]
            frame = torch.full((*lead, rows + 2, f + off + pad), 7.0, dtype=dtype, device="cuda")
            out = frame[..., 1:1 + rows, off:off + f]
            if gated:
                P.gated(xs, ws, b, act="gelu", out=out)
                pre = P.gated(x, w, b, act="gelu", keep_pre=True)[1]
                grads = P.gated_backward(ds, xs, ws, spread(pre), act="gelu")
            else:
                P.dense(xs, ws, b, rs, act="gelu", out=out)
                pre = P.dense(x, w, b, r, act="gelu", keep_pre=True)[1]
                grads = P.dense_backward(ds, xs, ws, spread(pre), act="gelu")
            v, e, _, _ = L.forward(x, w, b, r, "gelu", gated)
            L.check("y", out, v, e)
            keep = frame.clone()
            keep[..., 1:1 + rows, off:off + f] = 7.0
            assert bool((keep == 7.0).all())
            for name, got, (gv, ge) in zip(("dx", "dw", "db"), grads, L.backward(dy, x, w, pre, "gelu", gated)):
                L.check(name, got, gv, ge)


def test_population_views():
    """A layer of every member, as views into the asked population, and members interleaved within the rows."""
    P = _P()
    for dtype in TYPES:
        g = _gen(10)
        n, k, f, rows = 6, 20, 12, 7
        flat = _rand(g, n, k * f + f + 9, dtype=dtype, scale=0.2)
        w, b = flat[:, 3:3 + k * f].unflatten(1, (f, k)), flat[:, 3 + k * f:3 + k * f + f]
        x = _rand(g, rows, n, k, dtype=dtype).transpose(0, 1)  # [members, rows, in], members inside the rows
        out = torch.zeros(rows, n, f, dtype=dtype, device="cuda").transpose(0, 1)
        P.dense(x, w, b, act="tanh", out=out)
        v, e, _, _ = L.forward(x, w, b, None, "tanh")
        L.check("y", out, v, e)


def test_output_in_32_bits_and_in_place_residual():
    P = _P()
    for dtype in (BF, HF):
        for rows, k, f in ((5, 40, 33), (4, 2048, 64), (600, 256, 512)):
            x, w, b, r, _ = _case(11, dtype, None, rows, k, f, "none", residual=True)
            y = P.dense(x, w, b, r, out_dtype=SF)
            assert y.dtype == SF
            v, e, _, _ = L.forward(x, w, b, r, "none", dtype=SF)
            L.check("fp32", y, v, e)
            v, e, _, _ = L.forward(x, w, b, r, "silu")
            buf = r.clone()
            assert P.dense(x, w, b, buf, act="silu", out=buf) is buf
            L.check("in place", buf, v, e)
            h = P.gated(x, w[:f // 2 * 2], b[:f // 2 * 2], out_dtype=SF)
            v, e, _, _ = L.forward(x, w[:f // 2 * 2], b[:f // 2 * 2], None, "silu", True, dtype=SF)
            L.check("gated fp32", h, v, e)


@pytest.mark.parametrize("k,f", [(1031, 2051), (1032, 2056), (1024, 2048)])
def test_gradients_of_an_odd_address(k, f):
    """dy at an odd address with an activation: what the products read is dz, in the workspace."""
    P = _P()
    x, w, b, _, dy = _case(30, BF, None, 4100, k, f, "tanh")
    pre = P.dense(x, w, b, act="tanh", keep_pre=True)[1]
    moved = torch.empty(dy.numel() + 1, dtype=BF, device="cuda")[1:].view(dy.shape)
    moved.copy_(dy)
    for name, got, (v, bound) in zip(("dx", "dw", "db"), P.dense_backward(moved, x, w, pre, act="tanh"), L.backward(dy, x, w, pre, "tanh")):
        L.check(name, got, v, bound)


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan_stay_in_their_rows(dtype):
    P = _P()
    inf = float("inf")
    for rows, k, f in ((6, 33, 20), (200, 160, 150)):
        x, w, b, _, dy = _case(12, dtype, None, rows, k, f, "none")
        x[1, 3], x[2, 5], x[3, 0] = float("nan"), inf, -inf
        y = P.dense(x, w, b, act="relu")
        z = torch.matmul(x.double(), w.double().mT) + b.double()
        want = torch.where(z <= 0, 0.0, z).cpu()
        got = y.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got[2:4], want[2:4])  # infinities and zeros of relu
        fine = [i for i in range(rows) if i not in (1, 2, 3)]
        v, e, _, _ = L.forward(x[fine], w, b, None, "relu")
        L.check("others", y[fine], v, e)
        dy[1, 2] = float("nan")
        dx, _, _ = P.dense_backward(dy, x, w, None)
        assert bool(torch.isnan(dx[1]).all()) and bool(torch.isfinite(dx[2:]).all())


def test_far_activations():
    """Values where exponentials over- and underflow."""
    P = _P()
    for dtype in TYPES:
        z = torch.tensor([[-3e4, -200.0, -90.0, -20.0, -5.0, -1e-3, 0.0, 1e-4, 0.3, 4.0, 30.0, 95.0, 300.0, 3e4]], device="cuda").to(dtype)
        eye = torch.eye(z.shape[1], device="cuda").to(dtype)
        one = torch.ones(z.shape[1], 1, device="cuda").to(dtype)
        for act in ("relu", "tanh", "gelu", "silu"):
            y, pre = P.dense(z, eye, act=act, keep_pre=True)
            v, e, _, _ = L.forward(z, eye, None, None, act)
            L.check(act, y, v, e)
            dz = P.dense_backward(torch.ones_like(z), z, eye, pre, act=act, needs=(True, False, False))[0]
            (v, e), _, _ = L.backward(torch.ones_like(z), z, eye, pre, act)
            L.check(act + "'", dz, v, e)
            # a column of z alone: the gate's factor in a gated layer
            h = P.gated(one, torch.cat((z.mT, torch.ones_like(z.mT))), act=act)
            v, e, _, _ = L.forward(one, torch.cat((z.mT, torch.ones_like(z.mT))), None, None, act, True)
            L.check("gated " + act, h, v, e)


def test_gradients_against_differences():
    """fp32: the gradients of sum(c y) against central differences of the 64-bit form."""
    P = _P()
    for gated, act in ((False, "tanh"), (False, "gelu"), (True, "silu")):
        x, w, b, _, dy = _case(13, SF, None, 4, 6, 5, act, gated)
        if gated:
            pre = P.gated(x, w, b, act=act, keep_pre=True)[1]
            grads = P.gated_backward(dy, x, w, pre, act=act)
        else:
            pre = P.dense(x, w, b, act=act, keep_pre=True)[1]
            grads = P.dense_backward(dy, x, w, pre, act=act)

        def value(x, w, b):
            z = x @ w.mT + b
            if gated:
                f = z.shape[-1] // 2
                return (L.act(z[..., :f], act)[0] * z[..., f:] * L.d(dy)).sum()
            return (L.act(z, act)[0] * L.d(dy)).sum()

        args = [L.d(x), L.d(w), L.d(b)]
        for i, got in enumerate(grads):
            num = torch.zeros_like(args[i]).flatten()
            for j in range(num.numel()):
                for sign in (1, -1):
                    moved = [t.clone() for t in args]
                    moved[i].view(-1)[j] += sign * 1e-5
                    num[j] += sign * value(*moved) / 2e-5
            # differences: third derivatives times 1e-10 / 6 and 1e-16 / 1e-5 of the sums; fp32: pre's and the products'
            # roundings, well below 40 of them on sums of at most 10 terms of size 1
            assert (got.cpu().double().flatten() - num).abs().max() < 40 * L.U * 10 + 1e-8


def test_skipped_gradients_and_same_bits_twice():
    P = _P()
    x, w, b, _, dy = _case(14, BF, 3, 40, 56, 48, "gelu")
    pre = P.dense(x, w, b, act="gelu", keep_pre=True)[1]
    full = P.dense_backward(dy, x, w, pre, act="gelu")
    again = P.dense_backward(dy, x, w, pre, act="gelu")
    assert all(torch.equal(a, c) for a, c in zip(full, again))
    for i in range(3):
        needs = tuple(j == i for j in range(3))
        part = P.dense_backward(dy, x, w, pre, act="gelu", needs=needs)
        assert all((p is None) == (j != i) for j, p in enumerate(part))
        assert torch.equal(part[i], full[i])


def test_far_offsets():
    """Members whose matrices lie beyond 2^31 elements, 16 bits and 32."""
    P = _P()
    for dtype in (BF, SF):
        x, w, b, _, dy = _case(15, dtype, 2, 20, 24, 16, "tanh")
        far = (1 << 31) + 8
        flat = torch.empty(far + 24 * 20, dtype=dtype, device="cuda")
        xs = flat.as_strided((2, 20, 24), (far, 24, 1))
        xs.copy_(x)
        y, pre = P.dense(xs, w, b, act="tanh", keep_pre=True)
        v, e, _, _ = L.forward(x, w, b, None, "tanh")
        L.check("y", y, v, e)
        grads = P.dense_backward(dy, xs, w, pre, act="tanh")
        for name, got, (gv, ge) in zip(("dx", "dw", "db"), grads, L.backward(dy, x, w, pre, "tanh")):
            L.check(name, got, gv, ge)
        del flat, xs
        torch.cuda.empty_cache()


def test_other_stream_and_two_at_once():
    P = _P()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    # few rows and a long sum: both calls need a workspace
    x, w, b, _, _ = _case(16, BF, None, 40, 4096, 96, "tanh")
    x2 = x.flip(0).contiguous()
    torch.cuda.synchronize()
    ys = []
    for _ in range(8):
        ys.append((P.dense(x, w, b, act="tanh", stream=s1), P.dense(x2, w, b, act="tanh", stream=s2)))
    torch.cuda.synchronize()
    v, e, _, _ = L.forward(x, w, b, None, "tanh")
    for a, c in ys:
        L.check("y", a, v, e)
        L.check("y flipped", c.flip(0), v, e)


def test_captured_and_replayed():
    """Two graphs of forward and gradients, replayed in turn with eager work between, like the eager calls."""
    P = _P()
    graphs = []
    # split sums, fp32, the large tiles with parts, copies of ragged operands
    for seed, dtype, rows, k, f in ((17, BF, 48, 1024, 64), (18, SF, 33, 1024, 64), (19, HF, 4360, 1024, 4088), (20, BF, 2051, 2047, 2053)):
        x, w, b, _, dy = _case(seed, dtype, None, rows, k, f, "gelu")

        def step(x=x, w=w, b=b, dy=dy):
            y, pre = P.dense(x, w, b, act="gelu", keep_pre=True)
            return (y, pre, *P.dense_backward(dy, x, w, pre, act="gelu"))

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step()
        graphs.append((graph, outs, step, x))
    for turn in range(4):
        for graph, outs, step, x in graphs:
            x.mul_(-1.25)
            graph.replay()
            eager = step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(outs, eager)), turn
