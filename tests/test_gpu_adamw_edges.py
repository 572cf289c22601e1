"""AdamW at the ends of its arguments' ranges (marked gpu)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-40, 1e-45, 1.2e-38, 1e-8])
def test_smallest_eps(bits, eps):
    """Where moments and gradient are 0 the step is 0 / (0 + eps) = 0, however small eps is; elsewhere the first step moves
    by lr."""
    import paper_2212_04180_amd as P
    p = [torch.ones(600, device="cuda")]
    g = [torch.zeros(600, device="cuda")]
    g[0][::3] = -0.5
    s = P.adamw_state(p, bits)
    P.adamw(p, g, s["m"], s["v"], 1, lr=0.25, eps=eps, m_scale=s.get("m_scale"), v_scale=s.get("v_scale"))
    want = torch.where(g[0] == 0, 1.0, 1.25)
    # the step to 20 roundings and eps / 0.5, the sum to one
    assert bool(((p[0] - want).abs() <= 0.25 * (20 * 2.0 ** -24 + 2e-8) + 2.0 ** -23).all())
    assert bool((p[0][g[0] == 0] == 1.0).all())
