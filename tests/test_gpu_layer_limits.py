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
