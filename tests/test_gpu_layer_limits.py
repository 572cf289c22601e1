"""Layers at the limits of their sizes (marked gpu): offsets next to 2^31, counts of members beyond one launch."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _P():
    import paper_2212_04180_amd as P
    return P


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("k", [(1 << 31) - 1, (1 << 31) - 9])
def test_longest_rows(dtype, k):
    """One row of 2^31 - 1 inputs, NaN right behind it: a few ones among zeros, so that the sum is exact."""
    P = _P()
    x, w = (torch.zeros(k + 16, dtype=dtype, device="cuda") for _ in range(2))
    x[k:], w[k:] = float("nan"), float("nan")
    at = torch.tensor([0, 5, 70, 1 << 30, k - 70, k - 9, k - 2, k - 1], device="cuda")
    x[at] = 1.0
    w[at] = torch.arange(1, 9, device="cuda").to(dtype)
    y = P.dense(x[:k].view(1, k), w[:k].view(1, k), out_dtype=torch.float32)
    assert y.item() == 36.0
    del x, w
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_more_members_than_a_launch_holds(dtype):
    """2^24 + 5 members of one row: small whole numbers, so that every sum is exact."""
    P = _P()
    n = (1 << 24) + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, b, dy = (torch.randint(-3, 4, s, generator=g, device="cuda").to(dtype) for s in ((n, 1, 2), (n, 1, 2), (n, 1), (n, 1, 1)))
    y, pre = P.dense(x, w, b, act="relu", keep_pre=True)
    z = (x * w).sum(-1, keepdim=True) + b.unsqueeze(-1)
    assert torch.equal(pre, z) and torch.equal(y, z.clamp_min(0))
    dx, dw, db = P.dense_backward(dy, x, w, pre, act="relu")
    dz = dy * (z > 0)
    assert torch.equal(dx, dz * w) and torch.equal(dw, dz * x) and torch.equal(db, dz[:, 0])
    # one network: sums over the members
    y = P.dense(x, w[0], b[0], act="none")
    assert torch.equal(y, (x * w[0]).sum(-1, keepdim=True) + b[0])
    _, dw, db = P.dense_backward(dy, x, w[0], needs=(False, True, True))
    # whole numbers below 2^24 are exact in any order; the result is rounded once
    assert torch.equal(dw, (dy.double() * x.double()).sum(0).to(dtype)) and torch.equal(db, dy.double().sum((0, 1)).to(dtype))


def test_more_bias_gradients_than_a_launch_holds():
    """2^26 + 3 members of 65 rows: two chunks of rows each, added up by one workgroup a member."""
    P = _P()
    n = (1 << 26) + 3
    dy = torch.zeros(n, 65, 1, dtype=torch.bfloat16, device="cuda")
    a, b = (torch.arange(n, device="cuda") % p for p in (5, 7))
    dy[:, 0, 0], dy[:, 64, 0] = a.to(dy.dtype), b.to(dy.dtype)
    x = torch.zeros(65, 1, dtype=dy.dtype, device="cuda")
    w = torch.zeros(1, 1, 1, dtype=dy.dtype, device="cuda").expand(n, 1, 1)
    db = P.dense_backward(dy, x, w, needs=(False, False, True))[2]
    assert torch.equal(db[:, 0], (a + b).to(dy.dtype))
    del dy
    torch.cuda.empty_cache()
