"""Global gradient norm and clipping, against the definition in fp64."""
import numpy as np
import pytest
import torch

from paper_2506_01084_b200 import binding as zb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def clip(grads, outs, scale=1.0, max_norm=1.0):
    t = zb.grad_tensors(grads, outs)
    norm = torch.full((1,), 7.0, device=DEV)
    scratch = torch.full((max(8, zb.z2z_grad_clip_scratch_bytes(t)),), 255, dtype=torch.uint8, device=DEV)
    zb.z2z_grad_clip(t, scale, max_norm, norm, scratch)
    return norm.item()


def check(grads, outs, before, scale, max_norm, got):
    """The sum of squares: 7 additions in fp32 and the products' own rounding (8 U32 of a positive sum), halved by the
    root, then the norm's rounding.  The factor: quotient, sum and product (4 U32), then the product and the stored
    value's half step (which below the normal range is absolute)."""
    total = sum(float(b.double().pow(2).sum()) for b in before)
    norm = abs(scale) * np.sqrt(total)
    assert abs(got - norm) <= (4 + 1) * 1.01 * U32 * norm + 2.0 ** -149, (got, norm)
    factor = scale * min(1.0, max_norm / (norm + 1e-6))
    for b, o in zip(before, outs):
        if o is None:
            continue
        want = b.double() * factor
        off = (o.double() - want).abs()
        tol = ((5 + 4 + 1) * U32 + STEP[o.dtype]) * 1.01 * want.abs() + 2.0 ** -133
        assert bool((off <= tol).all()), (off.max().item(), b.shape, o.dtype)


def tensors(sizes, dtypes, shift=0, std=1.0, seed=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        dt = dtypes[i % len(dtypes)]
        flat = (torch.randn(n + shift, generator=g) * std).to(dt).to(DEV)
        out.append(flat[shift:])
    return out


@pytest.mark.parametrize("kind", ["same", "fp32", "bf16", "mixed"])
@pytest.mark.parametrize("dtypes", [[torch.float32], [torch.bfloat16], [torch.bfloat16, torch.float32]])
@pytest.mark.parametrize("shift", [0, 1, 2, 3, 5])
def test_types_and_alignment(kind, dtypes, shift):
    """Every combination of types; gradients that start off a 16-byte boundary, and outputs that start off it otherwise."""
    sizes = [1, 0, 7, 8, 9, 4095, 8192, 16384 + 7, 100003, 16384, 3]
    grads = tensors(sizes, dtypes, shift)
    before = [g.clone() for g in grads]
    if kind == "same":
        outs = grads
    else:
        dt = lambda i: {"fp32": torch.float32, "bf16": torch.bfloat16, "mixed": (torch.float32, torch.bfloat16)[i % 2]}[kind]  # noqa: E731
        flat = [torch.full((n + 12,), 7.0, dtype=dt(i), device=DEV) for i, n in enumerate(sizes)]
        outs = [f[i % 4:i % 4 + n] for i, (f, n) in enumerate(zip(flat, sizes))]
        if kind == "mixed":
            outs[4] = None
    got = clip(grads, outs, scale=0.5, max_norm=2.0)
    check(grads, outs, before, 0.5, 2.0, got)
    if kind != "same":
        for g, b in zip(grads, before):
            assert torch.equal(g, b)
        for i, (f, n) in enumerate(zip(flat, sizes)):                   # nothing around an output is touched
            assert bool((f[:i % 4] == 7).all()) and bool((f[i % 4 + n:] == 7).all())


def test_below_the_largest_norm_nothing_changes():
    grads = tensors([1000, 50000], [torch.bfloat16, torch.float32], std=1e-3)
    before = [g.clone() for g in grads]
    norm = clip(grads, grads, 1.0, 1.0)
    check(grads, grads, before, 1.0, 1.0, norm)
    assert norm < 1.0 and all(torch.equal(a, b) for a, b in zip(grads, before))
    outs = [torch.empty_like(g) for g in grads]
    clip(grads, outs, 1.0, float("inf"))
    assert all(torch.equal(a, b) for a, b in zip(outs, before))


@pytest.mark.parametrize("count", [0, 1, 511, 512, 513, 1500])
def test_many_tensors(count):
    grads = tensors([1 + (37 * i) % 900 for i in range(count)], [torch.float32, torch.bfloat16], seed=count)
    before = [g.clone() for g in grads]
    check(grads, grads, before, -2.0, 0.25, clip(grads, grads, -2.0, 0.25))


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e25, 3e38])
def test_squares_outside_the_range_of_fp32(size):
    g = [torch.full((999,), 0.0, device=DEV), torch.tensor([size, -size / 4, 0.0], device=DEV), torch.tensor([size / 8] * 11, device=DEV).bfloat16()]
    before = [x.clone() for x in g]
    outs = [torch.empty_like(x) for x in g]
    norm = clip(g, outs, 0.25, 1.0)
    check(g, outs, before, 0.25, 1.0, norm)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_norm_that_is_not_finite_leaves_the_outputs(bad):
    for place in (0, 4096, 70000):
        g = tensors([70001, 5000], [torch.bfloat16, torch.float32])
        g[0][place] = bad
        before = [x.clone() for x in g]
        outs = [torch.full_like(x, 3.0) for x in g]
        norm = clip(g, outs, 1.0, 0.5)
        assert not np.isfinite(norm) and np.isnan(norm) == np.isnan(bad)
        assert all(bool((o == 3.0).all()) for o in outs)
        clip(g, g, 1.0, 0.5)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(g, before))


def test_the_same_call_gives_the_same_bits_and_may_be_captured():
    grads = tensors([333333, 77, 1 << 20], [torch.bfloat16, torch.float32])
    outs = [torch.empty(g.numel(), device=DEV) for g in grads]
    t = zb.grad_tensors(grads, outs)
    norm, scratch = torch.empty(1, device=DEV), torch.empty(zb.z2z_grad_clip_scratch_bytes(t), dtype=torch.uint8, device=DEV)
    zb.z2z_grad_clip(t, 1.0, 1.0, norm, scratch)
    want = [norm.clone()] + [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zb.z2z_grad_clip(t, 1.0, 1.0, norm, scratch)
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, [norm] + outs))


def test_more_than_2_to_the_31_elements():
    n = (1 << 31) + 12345
    g = torch.full((n,), 0.0, dtype=torch.bfloat16, device=DEV)
    g[0], g[n - 1], g[1 << 31] = 3.0, 4.0, 12.0
    norm = clip([g], [g], 1.0, 1.0)
    assert abs(norm - 13.0) <= 13 * 5 * U32
    assert abs(g[n - 1].item() - 4 / 13) <= 2.0 ** -8 and abs(g[1 << 31].item() - 12 / 13) <= 2.0 ** -8 and g[1].item() == 0.0
