"""Pins of the cross entropy oracle: automatic differentiation in fp64, differences, rows that take no part."""
import numpy as np
import torch

from oracle import xent as ox


def case(seed=0, V=11, d=5, B=3, cap=4, N=17):
    g = np.random.default_rng(seed)
    seq = g.integers(0, B, N)
    n = [4, 0, 2]
    nvis = np.array([g.integers(0, n[b] + 1) for b in seq])
    target = np.array([g.integers(0, V + k) for k in nvis])
    return (g.normal(size=(N, d)), seq, nvis, g.normal(size=(V, d)), g.normal(size=(B, cap, d)), n, target), g.normal(size=N)


def test_against_automatic_differentiation():
    (h, seq, nvis, W, U, n, t), w = case()
    t[3] = -1                                               # no target
    t[5] = 11 + nvis[5]                                     # one the row does not see
    seq[7] = 3                                              # no sequence
    w[9] = 0.0
    got = ox.cross_entropy(h, seq, nvis, W, U, n, t, w)
    H, Wt, Ut = (torch.tensor(x, requires_grad=True) for x in (h, W, U))
    total = 0.0
    for r in range(len(t)):
        if r in (3, 5, 7):
            assert not got["live"][r] and got["loss"][r] == got["lse"][r] == 0.0
            continue
        l = torch.cat([Wt, Ut[seq[r], :nvis[r]]]) @ H[r]
        loss = torch.nn.functional.cross_entropy(l[None], torch.tensor([t[r]]))
        assert abs(loss.item() - got["loss"][r]) < 1e-12 and abs(torch.logsumexp(l, 0).item() - got["lse"][r]) < 1e-12
        total = total + w[r] * loss
    total.backward()
    for k, x in (("hidden", H), ("WU", Wt), ("Uh", Ut)):
        assert np.abs(got[k] - x.grad.numpy()).max() < 1e-12
        assert np.all(got["abs_" + k] >= np.abs(got[k]) - 1e-15)


def test_against_differences():
    args, w = case(1)
    got = ox.cross_entropy(*args, w)
    g = np.random.default_rng(5)
    for i, k in ((0, "hidden"), (3, "WU"), (4, "Uh")):
        step = g.normal(size=args[i].shape) * 1e-5
        up, down = ([a + s * step if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        diff = ((ox.cross_entropy(*up, w)["loss"] - ox.cross_entropy(*down, w)["loss"]) * w).sum() / 2
        assert abs(diff - (got[k] * step).sum()) < 1e-12
