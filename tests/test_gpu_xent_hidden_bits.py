"""Cross entropy of a bf16 session with fp32 gradients of the tables: the rows' gradient is off by its own rounding alone."""
import numpy as np
import pytest

from tests.test_gpu_xent import U32, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,d,N,cap,scratch", [(900, 96, 333, 300, "most"), (5000, 200, 40, 37, "least"), (20000, 64, 65, 0, "most")])
@pytest.mark.parametrize("mode", ["step", "autograd"])
def test_rows_gradient(V, d, N, cap, scratch, mode):
    c = Case("bf16", V=V, d=d, B=3, cap=cap, N=N, grads="fp32", scratch=scratch, causal=cap > 0, weights="mixed", seed=61)
    want = c.oracle()
    got = c.run(mode)
    c.check(got, want)
    # as Case.check has it for logits and probabilities; g in two parts of bf16, whose rest is below 2^-8 of 2^-8; sums
    # joined every few hundred products; half a step of bf16 for the stored value
    size = want["size"].max()
    e_l = ((d + 8) * 2 * U32 + 8 * U32) * size
    e_lse = e_l + 2 * U32 * np.abs(want["lse"]).max() + (64 + V / 64) * U32 + 2.0 ** -21
    x, y, mag = got["hidden"].double().cpu().numpy(), want["hidden"], want["abs_hidden"]
    tol = (2.0 ** -16 + e_l + e_lse + 2.0 ** -20 + (1024 + V / 256) * 2 * U32) * mag
    tol = tol + 2.0 ** -8 * (np.abs(y) + tol) * 1.01 + 1e-30
    off = np.abs(x - y)
    assert np.all(off <= tol), (off.max(), np.max(off / tol))
