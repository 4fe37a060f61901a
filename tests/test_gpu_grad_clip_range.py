"""Global norm of gradients most of which are zeros, tiny or huge, each size next to zeros and to ordinary values."""
import numpy as np
import pytest
import torch

from tests.test_gpu_grad_clip import DEV, check, clip

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [0.0, 2.0 ** -149, 1e-42, 1e-38, 1e-25, 1e-20, 9e-16, 1e-15, 1.1e-15, 1.0, 3e18, 1e19, 1.1e19, 1e30, 3e38])
@pytest.mark.parametrize("beside", [0.0, 1e-3, 1.0])
def test_sizes_side_by_side(dt, size, beside):
    if dt == torch.bfloat16 and size == 2.0 ** -149:
        size = 2.0 ** -133                       # its own smallest
    g = torch.full((40000,), 0.0, dtype=dt)
    g[:16] = g[100:1123] = size
    g[3] = -g[3]
    g[8000:9000:7] = size                        # one in a vector of zeros
    g[20000:30000] = beside
    g[30001] = size
    g = g.to(DEV)
    before = [g.clone()]
    out = torch.empty(40000, device=DEV)
    for scale in (1.0, 2.0 ** -7):
        total = float(before[0].double().pow(2).sum())
        got = clip([g], [out], scale, 0.5)
        if abs(scale) * np.sqrt(total) > 3.4e38:
            assert got == float("inf")
            continue
        check([g], [out], before, scale, 0.5, got)
