"""CPU oracle: one step of beam search over joint vocabularies (TEST INFRASTRUCTURE ONLY).

A live beam b offers its columns c with s = score_b + (l_c - lse_b) in fp64, a finished one offers itself; what has
s = -inf, once rounded to fp32, or NaN is no candidate.  The best `beams` of a group win, ordered by higher s, lower beam, higher logit,
lower column.  A parent's best continuation stays in the parent's slot, the others take the group's free slots in
order; slots without one are dead.

Pins: tests/test_oracle_operators.py (exhaustive enumeration on tiny vocabularies, one beam is greedy decoding,
every parent keeps its slot).
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np


def select(beams: int, rows: Sequence[np.ndarray], lse, scores, finished: Optional[Sequence[int]], eos: int):
    """rows[b]: the logits of beam b's columns.  Returns parent, code, score (fp64), finished, active per slot."""
    B = len(rows)
    parent, code, score = list(range(B)), [-1] * B, [-np.inf] * B
    ended, active = [1] * B, [0] * B
    for g in range(0, B, beams):
        cand = []
        for b in range(g, g + beams):
            if finished is not None and finished[b]:
                if scores[b] > -np.inf:
                    cand.append((-float(scores[b]), b, 0.0, -1))
                continue
            l = np.asarray(rows[b]).astype(np.float64)
            with np.errstate(invalid="ignore", over="ignore"):
                s = float(scores[b]) + (l - float(lse[b]))
                s = np.where(s.astype(np.float32) > -np.inf, s, -np.inf)         # (NaN, and sums below fp32's range)
            least = -np.partition(-s, beams - 1)[beams - 1] if s.size > beams else -np.inf
            for c in np.flatnonzero((s > -np.inf) & (s >= least)):            # what `beams` others beat cannot win
                cand.append((-s[c], b, -l[c], int(c)))
        cand.sort()
        won = cand[:beams]
        stay, move = {}, []
        for w in won:
            if w[1] in stay:
                move.append(w)
            else:
                stay[w[1]] = w
        free = [b for b in range(g, g + beams) if b not in stay]
        for slot, w in list(stay.items()) + list(zip(free, move)):
            fin = bool(finished is not None and finished[w[1]])
            parent[slot], code[slot], score[slot] = w[1], w[3], -w[0]
            ended[slot] = int(fin or (eos >= 0 and w[3] == eos))
            active[slot] = int(not fin)
    return parent, code, score, ended, active
