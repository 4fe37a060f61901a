"""Limits and temperatures that the distillation calls refuse on the host; no GPU is needed."""
import pytest
import torch

from paper_2506_01084_b200 import binding as zb


def test_wait_limit():
    with pytest.raises(zb.Z2ZError, match="ns < 0"):
        zb.z2z_set_distill_wait_limit(-1)
    zb.z2z_set_distill_wait_limit(10 ** 9)
    zb.z2z_set_distill_wait_limit(0)


@pytest.mark.parametrize("T", [1e-39, 2.9e-39, 3e-39, 4e-39, 4.2e-39])
def test_temperatures_whose_factor_is_not_finite(T):
    if torch.cuda.is_available():
        pytest.skip("the addresses here are made up: a call that was not refused must find no GPU")
    # 1 / T is finite from 2.94e-39 on, the exponents' factor log2(e) / T from 4.24e-39 on
    lib, at = zb.lib(), 4096
    for rc in (lib.z2z_distill_loss(at, 0, 2, 10, 10, None, at, at, 3, T, None, at, at, None, None),
               lib.z2z_distill_grad(at, 0, 2, 10, 10, None, at, at, 3, T, at, at, at, None)):
        assert rc == -1 and "temperature" in lib.z2z_last_error().decode()
