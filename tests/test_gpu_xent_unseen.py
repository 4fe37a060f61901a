"""Cross entropy: a row's gradient does not depend on hypertokens that it does not see, whatever they hold."""
import numpy as np
import pytest
import torch

from tests.test_gpu_xent import Case

pytestmark = pytest.mark.gpu
FORMS = [("bf16", None, "most"), ("bf16", None, "least"), ("bf16", "fp32", "most"), ("fp32", None, "most"), ("fp32", None, "least")]


def case(dtype, grads, scratch, d=72):
    c = Case(dtype, V=500, d=d, B=3, cap=300, counts=[300, 35, 64], N=160, grads=grads, scratch=scratch, causal=True, weights="mixed", seed=51)
    # nobody sees the last quarter of a sequence's entries
    c.nvis = torch.minimum(c.nvis, torch.tensor([225, 26, 48])[c.seq])
    c.target = torch.where(c.target >= 500 + c.nvis, c.target % 500, c.target)
    return c


@pytest.mark.parametrize("dtype,grads,scratch", FORMS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_entries_that_no_row_sees(dtype, grads, scratch, bad):
    """Such as those whose hyper-unembeddings have not been computed yet."""
    c = case(dtype, grads, scratch)
    want = c.oracle()
    for b, n in enumerate(c.counts):
        c.g_Uh[b, [225, 26, 48][b]:n] = bad
    for mode in ("step", "autograd"):
        c.check(c.run(mode), want)


@pytest.mark.parametrize("d", [72, 1160])
@pytest.mark.parametrize("dtype,grads,scratch", FORMS)
def test_entries_that_some_rows_see(dtype, grads, scratch, d):
    """Rows that see the entry have no gradient, those that do not see it keep theirs."""
    c = case(dtype, grads, scratch, d)
    want = c.oracle()
    c.g_Uh[0, 100, 3], c.g_Uh[2, 0, :] = float("nan"), float("nan")
    sees = ((c.seq == 0) & (c.nvis > 100)) | ((c.seq == 2) & (c.nvis > 0))
    live = torch.from_numpy(want["live"])
    assert int((sees & live).sum()) > 10 and int(((c.seq != 1) & ~sees & live).sum()) > 10
    for mode in ("step", "autograd"):
        got = c.run(mode)
        assert bool(got["loss"][sees & live].isnan().all())
        weighted = sees & live & (c.w != 0.0)
        assert bool(got["hidden"][weighted].isnan().any(1).all())
        for k in ("loss", "lse"):
            got[k][sees] = torch.from_numpy(want[k]).float().to(got[k])[sees]
        got["hidden"][sees] = torch.from_numpy(want["hidden"]).to(got["hidden"])[sees]
        for k in ("WU", "Uh"):                   # what is left to compare: the rows
            got[k] = torch.from_numpy(want[k]).to(got[k])
        for b, n in enumerate(c.counts):
            got["Uh"][b, n:] = c.gUh0.to(got["Uh"])[b, n:]
        c.check(got, want)
        assert np.isfinite(want["hidden"]).all()
