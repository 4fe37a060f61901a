"""The limit of the cross entropy's waits; no GPU is needed."""
import pytest

from paper_2506_01084_b200 import binding as zb


def test_wait_limit():
    with pytest.raises(zb.Z2ZError, match="ns < 0"):
        zb.z2z_set_xent_wait_limit(-1)
    zb.z2z_set_xent_wait_limit(10 ** 9)
    zb.z2z_set_xent_wait_limit(0)
