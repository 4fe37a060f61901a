"""Cross entropy: rows whose weight is 0 have gradient 0 whatever the tables hold."""
import pytest
import torch

from tests.test_gpu_xent import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,grads,scratch", [("bf16", None, "most"), ("bf16", None, "least"), ("bf16", "fp32", "most"), ("fp32", None, "most")])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["WU", "Uh"])
def test_a_table_that_is_not_finite(dtype, grads, scratch, bad, where):
    """An entry of W_U reaches all rows, one of U_h the rows of its sequence: those have no finite gradient then, unless their
    weight is 0; the rows of other sequences are as they were."""
    c = Case(dtype, V=600, d=72, B=3, cap=40, counts=[40, 17, 33], N=150, grads=grads, scratch=scratch, weights="mixed", seed=31)
    assert c.nvis is None
    light = c.w == 0.0
    assert 10 < int(light.sum()) < 100
    want = c.oracle()
    if where == "WU":
        c.WU[77, 5] = bad
        hit = torch.ones(150, dtype=torch.bool)
    else:
        c.g_Uh[1, 11, 5] = bad
        hit = c.seq == 1
    assert int((hit & light).sum()) > 3 and int((hit & ~light).sum()) > 3
    for mode in ("step", "autograd"):
        got = c.run(mode)
        h = got["hidden"].double().cpu()
        assert not bool(h[light].any()), "rows without weight"
        assert bool((~h[hit & ~light].isfinite()).any(1).all())
        # the rows that the entry does not reach
        for k in ("loss", "lse", "hidden"):
            got[k][hit] = torch.from_numpy(want[k]).to(got[k])[hit]
        for k in ("WU", "Uh"):
            got[k] = torch.from_numpy(want[k]).to(got[k])
        for b, n in enumerate(c.counts):
            got["Uh"][b, n:] = c.gUh0.to(got["Uh"])[b, n:]
        c.check(got, want)
