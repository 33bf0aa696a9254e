"""Group normalization with an activation at the ends of fp32's range."""
import pytest
import torch

import paper_2303_04769_amd as S
from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,W", [(4, 5), (90, 91)], ids=["registers", "pieces"])
def test_silu_of_values_at_the_end_of_the_range(H, W):
    """z / (1 + exp(-z)) and its derivative where exp(-z) is nothing, or infinite, and where z log2(e) is past fp32's range."""
    x = torch.randn(2, 1, H * W, 16, generator=torch.Generator().manual_seed(1)).to(DEV)
    dout = torch.randn(2, 1, H * W, 16, generator=torch.Generator().manual_seed(2)).to(DEV)
    beta = torch.zeros(16, device=DEV)
    ends = {1: float("inf"), 2: 3e38, 3: 2.4e38, 4: 2.3e38, 5: 100.0, 6: -100.0, 7: -2.3e38, 8: -3e38}
    for ch, b in ends.items():
        beta[ch] = b
    gamma = torch.ones(16, device=DEV)
    plan = S.GroupNorm(2, 16, H, W, 16, act="silu")
    out, stats, dx = torch.empty_like(x), torch.empty(2, 16, 2, device=DEV), torch.empty_like(x)
    plan.run(x, gamma, beta, out, stats)
    dg, db = torch.empty(16, device=DEV), torch.empty(16, device=DEV)
    plan.grad(x, gamma, beta, stats, dout, dx, dg, db)
    for ch, b in ends.items():
        if b > 50:
            assert bool((out[..., ch] == b).all() if b > 1e30 else (out[..., ch] > 90).all()), ch
        else:
            assert bool((out[..., ch] <= 0).all() and (out[..., ch] >= -1e-35).all()), ch
        if b != float("inf"):
            want = float(dout[..., ch].double().sum()) if b > 0 else 0.0
            assert abs(float(db[ch]) - want) <= 1e-4 * max(1.0, abs(want)), ch
            assert bool(torch.isfinite(dx[..., ch]).all()), ch
