"""Distillation of rows whose logits lie far from zero, against the fp64 oracle.

What all of a row's logits have in common must not reach a probability.  With x = (l - m) / T, u = 2^-24 and rows of C columns an
exponential's argument is off by 8 u |x| (the difference, the rounded factor log2 e / T, the product), whatever the level is, and
the exponential by 4 u more; the normaliser by e_s = (5 ln C + C / 256 + 40) u as in the tests of ordinary rows.  A column's q is
off by (8 |x| + 24) u + e_s of itself, p of a teacher's entry by (8 |y| + 24) u + (5 ln K + K + 40) u.  Up to an exponent of 2^12 the
factor of a bf16 gradient stands in the exponent, whose rounding, 2^-24 of it, adds 2^-12 ln 2."""
import numpy as np
import pytest
import torch

from oracle import distill as odis
from paper_2506_01084_b200 import binding as zb
from tests.test_gpu_distill import HALF, bounds, f64, u

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MASK = -1e30


def gradient_bound(l, ids, t, T, w, dt, want):
    C, K = l.size, ids.size
    x = (l - l.max()) / T
    q = np.exp(x)
    s = q.sum()
    e_s = (5 * np.log(C + 1) + C / 256 + 40) * u
    with np.errstate(invalid="ignore"):
        b = np.where(q > 0, q / s * ((8 * np.abs(x) + 24) * u + e_s + (2.0 ** -12 if dt == torch.bfloat16 else 0)), 0)
    y = (t - t.max()) / T
    p = np.exp(y) / np.exp(y).sum()
    np.add.at(b, ids, p * ((8 * np.abs(y) + 24) * u + (5 * np.log(K + 1) + 2 * K + 40) * u))
    return abs(w) * T * (b * 1.01 + 2.0 ** -126) + (3 * u + HALF[dt]) * np.abs(want)


def check(l, ids, t, T, w):
    """Row by row: all columns visible, weight w."""
    N, dt = l.shape[0], l.dtype
    g_l, gi, gt = l.to(DEV), torch.from_numpy(ids.astype(np.int32)).to(DEV), torch.from_numpy(t).to(DEV)
    gw = torch.full((N,), w, device=DEV)
    out = torch.full((4, N), 55.0, device=DEV)
    g = torch.full((2, *l.shape), 9.0, dtype=dt, device=DEV)
    zb.z2z_distill_loss(g_l, None, gi, gt, T, None, out[0], out[1])
    zb.z2z_distill_loss(g_l, None, gi, gt, T, gw, out[2], out[3], g[0])
    zb.z2z_distill_grad(g_l, None, gi, gt, T, out[1], gw, g[1])
    L = f64(l)
    w, T = float(np.float32(w)), float(np.float32(T))
    for r in range(N):
        tt = t[r].astype(np.float64)
        want_loss, want_lse, want = odis.row(L[r], ids[r], tt, T)
        want = want * w
        b_loss, b_lse, _ = bounds(L[r], ids[r], tt, T, w, dt, want)
        b_g = gradient_bound(L[r], ids[r], tt, T, w, dt, want)
        for a in (0, 2):
            assert abs(out[a + 1, r].item() - want_lse) <= b_lse, (r, a, out[a + 1, r].item(), want_lse, b_lse)
            assert abs(out[a, r].item() - want_loss) <= b_loss, (r, a, out[a, r].item(), want_loss, b_loss)
        for a in (0, 1):
            err = np.abs(f64(g[a, r]) - want)
            assert (err <= b_g).all(), (r, a, err.max(), (err / np.maximum(b_g, 1e-300)).max())


LEVELS = [0.0, 900.0, 3000.0, -3000.0, 1e5, -1e5, 2.0 ** 20, -(2.0 ** 20), -1e9, 3e9, -1e10, 1e12, 1e30, -1e30, 2e38, -8e37]


# clusters that hold the row, rows too long for that, and the persistent form
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1.0, 0.75])
@pytest.mark.parametrize("N,cols", [(16, 2003), (3, 1000003), (80, 70003)])
def test_distill_of_rows_far_from_zero(dt, T, N, cols):
    rng = np.random.default_rng(cols)
    l = np.zeros((N, cols), np.float32)
    for r in range(N):
        at = LEVELS[(r * (1 if N >= len(LEVELS) else 5) + 4) % len(LEVELS)]
        l[r] = at + rng.standard_normal(cols) * 2
        low = rng.random(cols) < 0.5                         # half of the columns far below, where the others are equal to rounding
        l[r, low] = at - 40 if abs(at) < 1e6 else at * (0.5 if at > 0 else 2.0)
        if r % 3 == 1:
            l[r, low & (rng.random(cols) < 0.5)] = MASK if at > MASK / 4 else 3 * at
    l[:, 7] = l.max(1)
    l = torch.from_numpy(np.clip(l, -3.3e38, 3.3e38)).to(dt)
    ids = np.stack([rng.choice(cols, 6, replace=False) for _ in range(N)])
    for r in range(N):                                       # (the teacher's columns have a probability)
        l[r, ids[r]] = l[r].max()
    t = (rng.standard_normal((N, 6)) * 2).astype(np.float32)
    check(l, ids, t, T, 0.375)
