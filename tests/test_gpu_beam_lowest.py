"""Beams whose sums leave fp32's range: a sum that is stored as -inf is that of a dead slot, and no candidate."""
import numpy as np
import pytest
import torch

from tests.test_gpu_beam import inputs, run_select
from tests.test_gpu_embed_scaled import session

pytestmark = pytest.mark.gpu
LOW = np.float32(np.finfo(np.float32).min)


@pytest.mark.parametrize("beams", [2, 4, 32])
@pytest.mark.parametrize("V", [5, 700, 9001])
def test_a_beam_that_takes_two_columns_of_the_lowest_value(V, beams):
    rng = np.random.default_rng(V + beams)
    B, cap = 3 * beams, 4
    n = [b % 5 for b in range(B)]
    cb = session(V, 8, cap, B, "fp32", [min(k, V - 1) for k in n])
    n = [min(k, V - 1) for k in n]
    l, lse, scores = inputs(rng, B, V, cap, n)
    for b in range(beams, B):                                # one column, or none, and masks
        l[b, :V + n[b]] = LOW
        if b % 2 and b < 2 * beams:
            l[b, b % V] = 1.0
        lse[b] = 1.0
    parent, code, score, ended, active = run_select(cb, beams, l, n, lse, scores, None, -1)
    assert all(np.isfinite(score[b]) == bool(active[b]) for b in range(B))
    # the next step, masked throughout: sums of two lowest values
    scores = np.array(score).astype(np.float32)
    assert (scores[np.array(active) == 1] > -np.inf).all() and (scores < -1e38).any()
    l[:, :] = LOW
    parent, code, score, ended, active = run_select(cb, beams, l, n, lse, scores, np.zeros(B, np.uint8), -1)
    assert all((np.float32(score[b]) > -np.inf) == bool(active[b]) for b in range(B))
