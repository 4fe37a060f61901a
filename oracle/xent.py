"""Cross entropy over the joint vocabulary and its gradients, in fp64, row by row from the definition."""
import numpy as np


def cross_entropy(hidden, seq, nvis, WU, Uh, n, target, weight=None):
    """hidden [N, d]; row r meets the rows of WU and then Uh[seq[r], :nvis[r]] (nvis None: all n of the sequence).
    Returns a dict: loss, lse [N]; gradients of sum(weight * loss): hidden [N, d], WU [V, d], Uh [B, cap, d]; and the
    same sums over magnitudes (abs_hidden, abs_WU, abs_Uh) and over p and [c = t] apart (for error bounds):
    a term's magnitude is |w| (p + [c = t]) |factor|.  Rows that take no part: zeros."""
    N, V = hidden.shape[0], WU.shape[0]
    B, cap = Uh.shape[0], Uh.shape[1]
    out = {"loss": np.zeros(N), "lse": np.zeros(N), "live": np.zeros(N, dtype=bool), "size": np.zeros(N)}
    for k, like in (("hidden", hidden), ("WU", WU), ("Uh", Uh)):
        out[k], out["abs_" + k] = np.zeros(like.shape), np.zeros(like.shape)
    for r in range(N):
        b = seq[r]
        if not 0 <= b < B:
            continue
        k = n[b] if nvis is None else min(max(nvis[r], 0), n[b])
        if not 0 <= target[r] < V + k:
            continue
        out["live"][r] = True
        M = np.concatenate([WU, Uh[b, :k]])
        with np.errstate(invalid="ignore", over="ignore"):
            l = M @ hidden[r]
            m = l.max()
            e = np.exp(l - m)
            tot = e.sum()
            out["lse"][r] = m + np.log(tot)
            out["loss"][r] = np.log(tot) + (m - l[target[r]])
            out["size"][r] = (np.abs(M) @ np.abs(hidden[r])).max()       # largest sum of magnitudes behind a logit
            w = 1.0 if weight is None else weight[r]
            if w == 0.0:
                continue
            p = e / tot
            one = np.zeros(V + k)
            one[target[r]] = 1.0
            for name, g, h, M_ in (("", w * (p - one), hidden[r], M), ("abs_", abs(w) * (p + one), np.abs(hidden[r]), np.abs(M))):
                out[name + "hidden"][r] = g @ M_
                out[name + "WU"] += np.outer(g[:V], h)
                out[name + "Uh"][b, :k] += np.outer(g[V:], h)
    return out
