"""Cross entropy kernels whose bounded waits give up: a limit of a few microseconds lets ordinary waits run out.  A block
leaves when the loads and products that it has under way have ended; the status tells of it, and later calls are as ever."""
import pytest
import torch

from paper_2506_01084_b200 import binding as zb
from tests.test_gpu_xent import Case

pytestmark = pytest.mark.gpu
# kept logits; pieces and g in parts; an fp32 session; few rows
FORMS = [dict(dtype="bf16", V=9000, d=1032, N=600, B=3, cap=300), dict(dtype="bf16", V=9000, d=1032, N=600, B=3, cap=300, grads="fp32", accumulate=True, scratch="least"),
         dict(dtype="fp32", V=3000, d=200, N=300, B=3, cap=40), dict(dtype="bf16", V=20000, d=2048, N=33, B=2, cap=20)]
LIMITS = (1, 1, 1000, 2000, 4000, 8000, 20000)


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("mode", ["step", "autograd"])
def test_waits_that_give_up(form, mode):
    c = Case(seed=71, causal=True, weights="mixed", **FORMS[form])
    want = c.run(mode)
    torch.cuda.synchronize()
    assert not any(v & zb.ST_WAIT_TIMEOUT for v in zb.z2z_status(c.cb)[0].tolist())
    try:
        for limit in LIMITS:
            zb.z2z_set_xent_wait_limit(limit)
            c.run(mode)
            torch.cuda.synchronize()
    finally:
        zb.z2z_set_xent_wait_limit(0)
    assert all(v & zb.ST_WAIT_TIMEOUT for v in zb.z2z_status(c.cb)[0].tolist())
    got = c.run(mode)
    for k in want:
        n = [slice(0, x) for x in c.counts]
        assert torch.equal(got[k], want[k]) if k != "Uh" else all(torch.equal(got[k][b, n[b]], want[k][b, n[b]]) for b in range(c.B)), k
