"""Cross entropy: probabilities of an fp32 session's step are as good as fp32 exponentials."""
import numpy as np
import pytest
import torch

from paper_2506_01084_b200 import binding as zb
from tests.test_gpu_xent import DEV, U32, session

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [3001, 8009])
@pytest.mark.parametrize("level", [0.9, 6.0, 40.0])
def test_rows_of_equal_logits_and_some_below(V, level):
    """The logits of row r are m_r, and m_r - a_r at every 128th column, exactly (one product with 1).  The sum of exponentials
    then has next to no error, and what lse and the differences to it lose to rounding shows in the p of those columns.  A
    column of the tables per row shows its p in W_U's gradient."""
    N, T = 1000, 0
    d = 8 + N
    g = torch.Generator().manual_seed(V)
    W, h = torch.zeros(V, d), torch.zeros(N, d)
    # (multiples of a step of fp32 at the largest of their sums, which are exact then)
    step = 2.0 ** -23 * 2.0 ** np.floor(np.log2(level + 1.0))
    m, a = (((torch.rand(N, generator=g, dtype=torch.float64) * 2 - 1) * level / step).round() * step,
            (torch.rand(N, generator=g, dtype=torch.float64) / step).round() * step)
    below = torch.arange(3, V, 128)
    W[:, 0], W[below, 1], h[:, 0], h[:, 1] = 1.0, -1.0, m, a
    assert torch.equal(h[:, 0].double(), m) and torch.equal(h[:, 1].double(), a) and torch.equal((h[:, 0] - h[:, 1]).double(), m - a)
    h[torch.arange(N), 8 + torch.arange(N)] = 1.0
    cb = session(V, d, 0, 1, "fp32", [0])
    target = torch.full((N,), T, dtype=torch.int32, device=DEV)
    loss, lse = torch.empty(2, N, device=DEV).unbind(0)
    gh, gW = torch.empty(N, d, device=DEV), torch.empty(V, d, device=DEV)
    scratch = torch.empty(zb.z2z_xent_scratch_bytes(cb.cfg, N, torch.float32)[1], dtype=torch.uint8, device=DEV)
    zb.z2z_xent_step(cb, h.to(DEV), torch.zeros(N, dtype=torch.int32, device=DEV), None, W.to(DEV), None, target, None, loss, lse, False, gh, gW, None,
                     scratch)
    m, a = m.numpy(), a.numpy()
    tot = V - len(below) + len(below) * np.exp(-a)
    p = gW.double().cpu().numpy()[:, 8:].T[:, below.numpy()]              # [row, column below]
    rel = p * (tot / np.exp(-a))[:, None] - 1.0
    # The sum: ones and 1 / 128 of its terms with errors of ex2 (2^-22 and its argument's half step), of which 1 / 16 step is
    # left; the joining of its fractions, 6 additions of a half step.  p: ex2's 2^-22, the product with its correction and
    # the correction's own, g's 24 bits, the tensor cores' sum of its parts (a step) and the stored value.
    tol = (0.1 + 6 + 4 + 6) * U32
    worst = np.abs(rel).max(1)
    assert worst.max() <= tol, (worst.max() / U32, tol / U32, int((worst > tol).sum()))
    want = np.log(tot)
    assert np.all(np.abs(loss.double().cpu().numpy() - want) <= 6.1 * U32 + 2 * U32 * want)
    assert np.all(np.abs(lse.double().cpu().numpy() - (m + want)) <= 6.1 * U32 + 2 * U32 * (np.abs(m) + want))
