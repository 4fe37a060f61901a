"""Cross entropy: the gradient at the target of rows that are sure of it, p - 1, at logits of any level."""
import math

import pytest
import torch

from paper_2506_01084_b200 import binding as zb
from tests.test_gpu_xent import DEV, U32, session

pytestmark = pytest.mark.gpu
LEVELS, GAPS = (0.0, 3.0, 20.0, 60.0, 300.0, 1000.0, -500.0), (8.0, 12.0, 15.0, 18.0)
V, CAP, T, D = 512, 1, 7, 80


@pytest.mark.parametrize("dtype,grads", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("mode", ["step", "step_least", "autograd"])
def test_the_target_of_a_confident_row(dtype, grads, mode):
    """Every logit of a row is its level, the target's lies a gap above (half of the rows: a base token, half: the hypertoken).
    Column 0 holds the level, 1 and 2 the gap; 3 is 1 in the token's row alone and 4 in the hypertoken's, so that a row's
    gradient is p_t - 1 in one of them; a column of its own for each row shows the same in the tables' gradients."""
    rows = [(a, b, h) for h in (False, True) for a in LEVELS for b in GAPS]
    N = len(rows)
    W, U, h = torch.zeros(V, D), torch.zeros(1, CAP, D), torch.zeros(N, D)
    W[:, 0] = U[0, :, 0] = 1.0
    W[T, 1] = U[0, 0, 2] = 1.0
    W[T, 3] = U[0, 0, 4] = 1.0
    for r, (level, gap, hyper) in enumerate(rows):
        h[r, 0], h[r, 2 if hyper else 1], h[r, 10 + r] = level, gap, 1.0
    cb = session(V, D, CAP, 1, "bf16" if dtype == torch.bfloat16 else "fp32", [1])
    target = torch.tensor([V if hyper else T for _, _, hyper in rows], dtype=torch.int32, device=DEV)
    seq = torch.zeros(N, dtype=torch.int32, device=DEV)
    args = (cb, h.to(DEV, dtype), seq, None, W.to(DEV, dtype), U.to(DEV, dtype), target)
    assert torch.equal(args[1].float().cpu(), h)
    loss, lse = torch.empty(2, N, device=DEV).unbind(0)
    gh = torch.empty(N, D, dtype=dtype, device=DEV)
    gW, gU = torch.empty(V, D, dtype=grads, device=DEV), torch.empty(1, CAP, D, dtype=grads, device=DEV)
    scratch = torch.empty(zb.z2z_xent_scratch_bytes(cb.cfg, N, grads)[0 if mode == "step_least" else 1], dtype=torch.uint8, device=DEV)
    if mode == "autograd":
        zb.z2z_xent_loss(*args, loss, lse, scratch)
        zb.z2z_xent_grad(*args, lse, None, False, gh, gW, gU, scratch)
    else:
        zb.z2z_xent_step(*args, None, loss, lse, False, gh, gW, gU, scratch)
    for r, (level, gap, hyper) in enumerate(rows):
        others = V * math.exp(-gap)              # (a token and the hypertoken less the target)
        exact = -others / (1.0 + others)
        # the sum of exponentials: at most 48 of its additions and merges have the target's 1 in them, ex2 is good to
        # 2^-22; the loss alone gives lse rounded to fp32
        off = 48 * U32 + abs(exact) * 2.0 ** -20 + (abs(level + gap) * U32 if mode == "autograd" else 0.0)
        # roundings to bf16: g's where gradients are bf16 and for a row's gradient, and the stored values'
        half = lambda dt: 2.0 ** -8 if dt == torch.bfloat16 else U32  # noqa: E731
        at = gU[0, 0] if hyper else gW[T]
        for name, got, dt in (("hidden", gh[r, 4 if hyper else 3], dtype), ("table", at[10 + r], grads)):
            tol = 1.01 * (off + abs(exact) * (half(dt) + 2 * half(dt if name == "hidden" else grads)))
            assert abs(got.item() - exact) <= tol, (name, level, gap, hyper, got.item(), exact, tol)
