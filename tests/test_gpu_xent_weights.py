"""Cross entropy: a weight that is not finite reaches its own row's gradient and the tables', and nothing else."""
import numpy as np
import pytest
import torch

from tests.test_gpu_xent import Case

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("dtype,grads,scratch", [("bf16", None, "most"), ("bf16", None, "least"), ("bf16", "fp32", "most"), ("fp32", None, "most")])
@pytest.mark.parametrize("bad", [[NAN], [INF], [-INF], [NAN, INF, -INF]])
def test_other_rows_keep_their_gradients(dtype, grads, scratch, bad):
    c = Case(dtype, V=500, d=72, B=3, cap=40, N=120, grads=grads, scratch=scratch, weights="mixed", causal=True, seed=41)
    rows = torch.arange(3, 3 + 17 * len(bad), 17)
    c.w[rows] = 0.0
    want = c.oracle()                            # (the losses do not depend on weights)
    c.w[rows] = torch.tensor(bad)
    for mode in ("step", "autograd"):
        got = c.run(mode)
        assert bool((~got["hidden"][rows].isfinite()).any(1).all())
        assert not bool(got["WU"].isfinite().any())
        got["hidden"][rows] = 0.0
        for k in ("WU", "Uh"):                   # what is left to compare: the rows
            got[k] = torch.from_numpy(want[k]).to(got[k])
            for b, n in enumerate(c.counts):
                if k == "Uh":
                    got[k][b, n:] = c.gUh0.to(got[k])[b, n:]
        c.check(got, want)


@pytest.mark.parametrize("others", [0.0, NAN])
def test_no_weight_is_finite_and_not_zero(others):
    c = Case("bf16", V=300, d=64, B=2, cap=20, N=40, weights="none", seed=42)
    c.w = torch.full((40,), others)
    c.w[5] = INF
    for mode in ("step", "autograd"):
        got = c.run(mode)
        lost = (~got["hidden"].isfinite()).any(1).cpu().numpy()
        assert np.array_equal(lost, np.isnan(c.w.numpy()) | np.isinf(c.w.numpy()))
        assert not bool(got["hidden"][~torch.from_numpy(lost)].any())
