"""The selection's oracle where sums leave fp32's range (they are stored in fp32): no live slot has a score of -inf."""
import numpy as np

from oracle import beam as obeam

LOW = np.finfo(np.float32).min


def test_sums_below_the_range_of_fp32_are_no_candidates():
    rows = [np.full(4, LOW, np.float32), np.full(4, LOW, np.float32)]
    lse, scores = [0.0, 0.0], np.array([0.0, LOW], np.float32)
    parent, code, score, ended, active = obeam.select(2, rows, lse, scores, None, -1)
    assert parent == [0, 0] and code == [0, 1] and active == [1, 1]              # the first beam's; the second's sums are 2 LOW
    scores[0] = LOW
    parent, code, score, ended, active = obeam.select(2, rows, lse, scores, None, -1)
    assert code == [-1, -1] and score == [-np.inf] * 2 and ended == [1, 1] and active == [0, 0]
    # half a step below the lowest value still rounds to it
    rows[0][2] = -2.0 ** 102
    parent, code, score, ended, active = obeam.select(2, rows, lse, scores, None, -1)
    assert code == [2, -1] and active == [1, 0] and np.float32(score[0]) == LOW
