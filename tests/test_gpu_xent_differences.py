"""Cross entropy: gradients along a direction against differences of losses, with bounds that a gradient of zeros or of
the other sign does not meet."""
import numpy as np
import pytest
import torch

from oracle import xent as ox
from tests.test_gpu_xent import U32, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["step", "autograd"])
@pytest.mark.parametrize("dtype,grads", [("fp32", None), ("bf16", "fp32"), ("bf16", None)])
def test_gradients_along_a_direction(dtype, grads, mode):
    """The direction is the sign of the gradient, so that all terms of <gradient, direction> add up.  Differences: of the
    oracle's losses in fp64, at two widths, extrapolated; what is left of their error shows in how far the two widths are apart."""
    c = Case(dtype, V=120, d=32, B=2, cap=16, N=40, grads=grads, weights="mixed", causal=True, seed=21)
    got, want = c.run(mode), c.oracle()
    f = lambda t: t.double().numpy()  # noqa: E731
    base = {"hidden": f(c.hidden), "WU": f(c.WU), "Uh": f(c.Uh)}
    w = f(c.w)

    def total(at):
        o = ox.cross_entropy(at["hidden"], c.seq.numpy(), c.nvis.numpy(), at["WU"], at["Uh"], c.counts, c.target.numpy(), w)
        return (o["loss"] * w).sum()

    for k in base:
        grad = got[k].double().cpu().numpy()
        if k == "Uh":
            for b, n in enumerate(c.counts):
                grad[b, n:] = 0.0
        step = np.sign(want[k])
        slope = lambda h: (total(dict(base, **{k: base[k] + h * step})) - total(dict(base, **{k: base[k] - h * step}))) / (2 * h)  # noqa: E731
        wide, narrow = slope(2.0 ** -11), slope(2.0 ** -12)
        diff = narrow + (narrow - wide) / 3
        along = float((grad * step).sum())
        # what Case.check allows for an element, all in one direction
        size = want["size"].max()
        e_l = ((c.d + 8) * 2 * U32 + 8 * U32) * size
        e_lse = e_l + 2 * U32 * np.abs(want["lse"]).max() + (64 + c.V / 64) * U32 + 2.0 ** -21
        half = 2.0 ** -8 if k == "hidden" and c.dt == torch.bfloat16 or c.gt == c.dt == torch.bfloat16 else 2.0 ** -23
        rel = half + e_l + e_lse + 2.0 ** -20 + (2.0 ** -12 if half == 2.0 ** -8 else 0.0) + (c.V + 16) * 2 * U32
        tol = rel * want["abs_" + k].sum() + 1.01 * half * np.abs(want[k]).sum() + abs(narrow - wide) + 1e-9
        assert abs(along - diff) <= tol, (k, along, diff, tol)
        assert tol < 0.2 * abs(diff), (k, tol, diff)
        assert abs(diff - (want[k] * step).sum()) <= abs(narrow - wide) + 1e-9
