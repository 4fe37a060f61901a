"""Distillation kernels whose bounded waits give up: a limit of a few microseconds lets ordinary waits run out.  Whatever a
call then leaves of a row is what it leaves without the limit, bit for bit, or NaN throughout."""
import numpy as np
import pytest
import torch

from paper_2506_01084_b200 import binding as zb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(dt, N, cols, K):
    g = torch.Generator(device=DEV)
    g.manual_seed(N + cols)
    l = (torch.randn(N, cols, generator=g, device=DEV) * 2).to(dt)
    n = (cols - torch.randint(0, cols // 2, (N,), generator=g, device=DEV)).int()
    n[1], n[2] = 0, cols
    ids = torch.randint(0, cols, (N, K), generator=g, device=DEV).int()
    ids[3] = -1
    t = torch.randn(N, K, generator=g, device=DEV) * 2
    w = torch.rand(N, generator=g, device=DEV) + 0.1
    w[4] = 0.0
    return (l, n, ids, t, 1.5), w


def forms(args, w, lse):
    """Results of the loss alone, of the loss with the gradient, and of the backward pass on its own."""
    l = args[0]
    N = l.shape[0]
    out = torch.full((4, N), 55.0, device=DEV)
    g = torch.full((2, *l.shape), 9.0, dtype=l.dtype, device=DEV)
    zb.z2z_distill_loss(*args, None, out[0], out[1])
    zb.z2z_distill_loss(*args, w, out[2], out[3], g[0])
    zb.z2z_distill_grad(*args, lse, w, g[1])
    torch.cuda.synchronize()
    return out, g


# clusters of one, two, four and eight blocks, with one row and with several each
@pytest.mark.parametrize("dt,N,cols", [(torch.bfloat16, 296, 70003), (torch.float32, 222, 132347), (torch.float32, 80, 132352), (torch.float32, 111, 262147),
                                       (torch.float32, 80, 300007), (torch.bfloat16, 148, 580003)])
def test_rows_of_a_wait_that_gave_up_are_nan(dt, N, cols):
    args, w = inputs(dt, N, cols, 40)
    lse = torch.zeros(N, device=DEV)                         # (the backward pass reads nothing of it but -inf)
    want, want_g = forms(args, w, lse)
    assert not want.isnan().any() and not want_g.isnan().any()
    given_up = 0
    try:
        for limit in (1, 1, 1000, 1500, 2500, 4000, 8000, 30000):
            zb.z2z_set_distill_wait_limit(limit)
            got, got_g = forms(args, w, lse)
            for a in (0, 2):
                lost = got[a].isnan()
                assert torch.equal(lost, got[a + 1].isnan())
                assert torch.equal(got[a][~lost], want[a][~lost]) and torch.equal(got[a + 1][~lost], want[a + 1][~lost])
                given_up += int(lost.sum())
            for a in (0, 1):
                lost = got_g[a].isnan().any(1)
                assert torch.equal(lost, got_g[a].isnan().all(1))
                assert torch.equal(got_g[a][~lost], want_g[a][~lost])
                if a == 0:
                    assert torch.equal(lost, got[2].isnan())
    finally:
        zb.z2z_set_distill_wait_limit(0)
    assert given_up > 0
    got, got_g = forms(args, w, lse)
    assert torch.equal(got, want) and torch.equal(got_g, want_g)
