"""Teachers and students whose logits are the lowest or the largest of their type, against the fp64 oracle.

Bounds, with u = 2^-24: the normaliser of C columns is off by e_s = (5 ln C + C / 256 + 40) u as in the tests of ordinary rows;
a bracket log p - log q of ordinary size (below 40 here) by 64 roundings of it, one of some 1e38 by 2^-18 of itself; a gradient by
e_s, 64 u, and for bf16 the rounding of an exponent, 2^-12, of its q, and one rounding to its type."""
import numpy as np
import pytest
import torch

from oracle import distill as odis
from paper_2506_01084_b200 import binding as zb
from tests.test_gpu_distill import HALF, f64, u

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LOW, TOP = float(np.finfo(np.float32).min), float(np.finfo(np.float32).max)


def check(l, ids, t, T):
    N, dt = l.shape[0], l.dtype
    g_l, gi, gt = l.to(DEV), torch.from_numpy(ids.astype(np.int32)).to(DEV), torch.from_numpy(t.astype(np.float32)).to(DEV)
    out = torch.full((4, N), 55.0, device=DEV)
    g = torch.full((2, *l.shape), 9.0, dtype=dt, device=DEV)
    zb.z2z_distill_loss(g_l, None, gi, gt, T, None, out[0], out[1])
    zb.z2z_distill_loss(g_l, None, gi, gt, T, None, out[2], out[3], g[0])
    zb.z2z_distill_grad(g_l, None, gi, gt, T, out[1], torch.ones(N, device=DEV), g[1])
    L = f64(l)
    for r in range(N):
        want_loss, want_lse, want = odis.row(L[r], ids[r], t[r].astype(np.float32).astype(np.float64), T)
        e_s = (5 * np.log(L.shape[1]) + L.shape[1] / 256 + 40) * u
        for a in (0, 2):
            assert abs(out[a + 1, r].item() - want_lse) <= e_s + 4 * u * (40 + abs(want_lse))
            assert abs(out[a, r].item() - want_loss) <= T * T * (e_s + 64 * 40 * u) + 2.0 ** -18 * abs(want_loss), (r, out[a, r].item(), want_loss)
        q = np.exp((L[r] - L[r].max()) / T)
        b = T * (e_s + 64 * u + (2.0 ** -12 * q / q.sum() if dt == torch.bfloat16 else 0)) + HALF[dt] * np.abs(want)
        for a in (0, 1):
            assert (np.abs(f64(g[a, r]) - want) <= b).all(), r


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1.0, 2.5])
@pytest.mark.parametrize("N,cols", [(8, 1003), (80, 70003)])
def test_teachers_logits_at_the_ends_of_the_type(dt, T, N, cols):
    rng = np.random.default_rng(cols)
    l = (torch.from_numpy(rng.standard_normal((N, cols)).astype(np.float32))).to(dt)
    ids = np.stack([rng.choice(cols, 5, replace=False) for _ in range(N)])
    t = rng.standard_normal((N, 5))
    t[0] = LOW                                               # equal: a fifth each
    t[1] = TOP
    t[2, 1:] = LOW
    t[3, :4] = [LOW, TOP, 0.0, -np.inf]
    t[4] = -3e38
    t[5, 0] = TOP
    t[6] = [-1e30, -1e30, LOW, LOW, -np.inf]
    check(l, ids, t, T)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1.0, 2.0])
@pytest.mark.parametrize("N,cols", [(8, 1003), (80, 70003)])
def test_teachers_columns_that_the_student_masks_with_the_lowest_value(dt, T, N, cols):
    rng = np.random.default_rng(cols + 1)
    l = (torch.from_numpy(rng.standard_normal((N, cols)).astype(np.float32))).to(dt)
    ids = np.stack([rng.choice(cols, 6, replace=False) for _ in range(N)])
    t = rng.standard_normal((N, 6)) * 0.1                    # a sixth each, about
    low = torch.finfo(dt).min
    l[0, ids[0, 2]] = low
    l[1, ids[1, :2]] = low
    l[3] = low
    l[3, ids[3, 5]] = 2.0                                    # one column left
    t[3, :5] -= 20.0
    l[4] = low
    l[4, (ids[4, 0] + 1) % cols] = -5.0
    ids[4, 1] = (ids[4, 0] + 1) % cols
    t[4] = [-1.0, 0.0, -np.inf, -np.inf, -np.inf, -np.inf]
    check(l, ids, t, T)
