"""Pins of the oracles of the scaled lookup's gradient, distillation and beam selection (CPU)."""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import beam as obeam, distill as odis, embedding as oemb


def test_lookup_gradient_is_the_adjoint_of_the_lookup():
    rng = np.random.default_rng(0)
    V, cap, B, d, N = 11, 5, 3, 4, 60
    n = [5, 0, 3]
    seq = rng.integers(0, B, N)
    codes = np.array([rng.integers(0, V + n[b]) for b in seq])
    codes[::7] = -1
    g = rng.standard_normal((N, d))
    dW, dE, cW, cE, aW, aE = oemb.lookup_grad(codes, seq, g, V, cap, B, n, 1.7)
    assert cW.sum() + cE.sum() == (codes >= 0).sum() and (aW >= np.abs(dW) - 1e-12).all() and (aE >= np.abs(dE) - 1e-12).all()
    for _ in range(5):                                       # <g, L(W, E)> = <L*(g), (W, E)> for every pair of tables
        W, E = rng.standard_normal((V, d)), rng.standard_normal((B, cap, d))
        out, bad = oemb.lookup_scaled(codes, seq, W, E, n, 1.7)
        assert not bad
        assert math.isclose((g * out).sum(), (dW * W).sum() + (dE * E).sum(), rel_tol=1e-12, abs_tol=1e-12)


def test_distillation_gradient_by_differences_and_by_automatic_differentiation():
    rng = np.random.default_rng(1)
    C, K, T = 13, 5, 1.7
    l = rng.standard_normal(C) * 2
    ids = np.array([3, 12, 3, -1, 7])                        # a column named twice, an entry that is absent
    t = rng.standard_normal(K) * 2
    loss, lse, grad = odis.row(l, ids, t, T)
    assert math.isclose(lse, math.log(np.exp(l / T).sum()), rel_tol=1e-14)
    for c in range(C):
        e = np.zeros(C); e[c] = 1e-6
        diff = (odis.row(l + e, ids, t, T)[0] - odis.row(l - e, ids, t, T)[0]) / 2e-6
        assert abs(diff - grad[c]) < 1e-8
    x = torch.tensor(l, requires_grad=True)
    keep = torch.tensor(ids >= 0)
    logp = torch.log_softmax(torch.tensor(t)[keep] / T, 0)
    logq = torch.log_softmax(x / T, 0)[torch.tensor(ids)[keep]]
    want = T * T * (logp.exp() * (logp - logq)).sum()
    want.backward()
    assert math.isclose(want.item(), loss, rel_tol=1e-12)
    assert np.abs(x.grad.numpy() - grad).max() < 1e-13
    assert abs(grad.sum()) < 1e-13                           # a shift of all logits changes nothing


def test_distillation_of_the_teacher_itself_and_empty_rows():
    l = np.array([0.3, -1.0, 2.0])
    loss, _, grad = odis.row(l, [0, 1, 2], l, 2.0)
    assert abs(loss) < 1e-14 and np.abs(grad).max() < 1e-14
    assert odis.row(l, [-1, 9], [1.0, 1.0], 1.0)[0] == 0.0 and not odis.row(l, [-1, 9], [1.0, 1.0], 1.0)[2].any()
    loss, lse, grad = odis.row(np.full(3, -np.inf), [0], [1.0], 1.0)
    assert loss == 0.0 and lse == -np.inf and not grad.any()
    loss, lse, grad = odis.row(np.array([-np.inf, 1.0]), [1], [1.0], 1.0)
    assert loss == 0.0 and lse == 1.0 and not grad.any()     # all of the student's mass where the teacher's is


@pytest.mark.parametrize("beams", [1, 2, 3])
def test_beam_selection_by_enumeration(beams):
    rng = np.random.default_rng(beams)
    for _ in range(50):
        C = [int(c) for c in rng.integers(1, 5, beams)]
        rows = [rng.integers(-2, 3, c).astype(np.float32) for c in C]           # many ties
        scores = rng.integers(-3, 1, beams).astype(np.float32)
        scores[rng.random(beams) < 0.2] = -np.inf
        fin = (rng.random(beams) < 0.3).astype(np.uint8)
        lse = rng.integers(0, 3, beams).astype(np.float32)
        parent, code, score, ended, active = obeam.select(beams, rows, lse, scores, fin, 1)
        every = []
        for b in range(beams):
            if fin[b]:
                every.append((float(scores[b]), b, 0.0, -1))
            else:
                every += [(float(scores[b]) + (float(x) - float(lse[b])), b, float(x), c) for c, x in enumerate(rows[b])]
        every = [e for e in every if e[0] > -np.inf]
        # the winners: a set of the right size that no candidate left out is ahead of
        better = lambda a, b: a[0] > b[0] or (a[0] == b[0] and (a[1] < b[1] or (a[1] == b[1] and (a[2] > b[2] or (a[2] == b[2] and a[3] < b[3])))))  # noqa: E731
        got = {(parent[i], code[i]) for i in range(beams) if score[i] > -np.inf}
        assert len(got) == min(beams, len(every)) == sum(s > -np.inf for s in score)
        for e in every:
            ahead = sum(better(o, e) for o in every)
            assert ((e[1], e[3]) in got) == (ahead < beams)
        for i in range(beams):
            assert parent[parent[i]] == parent[i]            # a parent keeps its slot
            if score[i] == -np.inf:
                assert parent[i] == i and code[i] == -1 and ended[i] and not active[i]
            else:
                assert active[i] == (not fin[parent[i]]) and ended[i] == (fin[parent[i]] or code[i] == 1)


def test_one_beam_is_greedy():
    rng = np.random.default_rng(5)
    for _ in range(20):
        l = rng.integers(0, 4, 9).astype(np.float32)
        parent, code, score, ended, active = obeam.select(1, [l], [2.0], [0.5], None, -1)
        assert parent == [0] and code == [int(np.argmax(l))] and score == [0.5 + (float(l.max()) - 2.0)] and ended == [0] and active == [1]
