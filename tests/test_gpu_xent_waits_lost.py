"""Cross entropy kernels whose bounded waits give up: whatever a call then leaves is what it leaves without the limit, bit for
bit, or NaN."""
import pytest
import torch

from paper_2506_01084_b200 import binding as zb
from tests.test_gpu_xent import Case
from tests.test_gpu_xent_waits import FORMS, LIMITS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("mode", ["step", "autograd"])
def test_what_did_not_come_is_nan(form, mode):
    c = Case(seed=72, causal=True, weights="mixed", **FORMS[form])
    want = c.run(mode)
    own = {k: ~v.isnan() for k, v in want.items()}
    for b, n in enumerate(c.counts):
        own["Uh"][b, n:] = False                 # (the caller's)
    assert all(bool(own[k].all()) for k in own if k != "Uh")
    lost = 0
    try:
        for limit in LIMITS:
            zb.z2z_set_xent_wait_limit(limit)
            got = c.run(mode)
            torch.cuda.synchronize()
            for k in want:
                nan = got[k].isnan()
                assert bool((nan | (got[k] == want[k]) | ~own[k]).all()), (k, limit)
                lost += int((nan & own[k]).sum())
    finally:
        zb.z2z_set_xent_wait_limit(0)
    assert lost > 0
