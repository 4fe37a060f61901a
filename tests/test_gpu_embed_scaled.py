"""Scaled mixed-stream lookup and its gradient by sorted tokens against the fp64 oracle.

Bounds: the lookup takes one product in fp32 and one rounding.  A gradient row of m terms is a sum in fp32, in
whatever order: |error| <= (m + 4) 2^-24 sum |scale g| (m - 1 additions, the product with the scale, the addition to
the old value), and one rounding to the table's type."""
import numpy as np
import pytest
import torch

from oracle import embedding as oemb
from paper_2506_01084_b200 import binding as zb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def session(V, d, cap, B, dtype, n):
    """A session whose sequence b has n[b] hypertokens: a prompt of n[b] + 1 distinct tokens."""
    cb = zb.Codebook(zb.make_config(V, d, 3, cap, B, dtype, 0, 1, 8), DEV)
    T = max(n) + 1
    assert T <= V
    tok = ((np.arange(T)[None, :] + 3 * np.arange(B)[:, None]) % V).astype(np.int32)
    lens = torch.tensor([k + 1 if k else 0 for k in n], dtype=torch.int32, device=DEV)
    codes = torch.zeros(B, T, dtype=torch.int32, device=DEV)
    zb.z2z_lzw_encode(cb, torch.from_numpy(tok).to(DEV), lens, codes, torch.zeros(B, dtype=torch.int32, device=DEV))
    assert zb.z2z_status(cb)[1].tolist() == list(n)
    return cb


def stream(rng, N, V, B, n, share=0.5, few=None):
    seq = np.sort(rng.integers(0, B, N)).astype(np.int32)
    codes = rng.integers(0, few or V, N)
    for r in range(N):
        if n[seq[r]] > 0 and rng.random() < share:
            codes[r] = V + rng.integers(0, n[seq[r]])
    codes[rng.random(N) < 0.1] = -1
    return codes.astype(np.int32), seq


def gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def f64(t):
    return t.detach().cpu().double().numpy()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [8, 40, 264, 1000, 4096])
@pytest.mark.parametrize("N", [1, 3, 77, 1500])
def test_lookup_scaled(dtype, d, N):
    rng = np.random.default_rng(d + N)
    V, cap, B = 300, 20, 4
    n = [20, 0, 7, 13]
    cb = session(V, d, cap, B, dtype, n)
    W = torch.from_numpy(rng.standard_normal((V, d)).astype(np.float32)).to(DT[dtype]).to(DEV)
    E = torch.from_numpy(rng.standard_normal((B, cap, d)).astype(np.float32)).to(DT[dtype]).to(DEV)
    codes, seq = stream(rng, N, V, B, n)
    if N > 50:
        codes[10], codes[11], codes[12] = V + n[seq[10]], -9, 1 << 30           # they name nothing
        seq[20] = -1                                                            # no sequence
        seq[21] = B
    out = torch.full((N, d), 7.0, dtype=DT[dtype], device=DEV)
    for scale in (1.0, 31.625, -0.3, 0.0):
        zb.z2z_embed_lookup_scaled(cb, gpu(codes), gpu(seq), W, E, scale, out)
        s32 = float(np.float32(scale))
        ok = (seq >= 0) & (seq < B)
        want, bad = oemb.lookup_scaled(np.where(ok, codes, -1), np.where(ok, seq, 0), f64(W), f64(E), n, s32)
        assert (np.abs(f64(out) - want) <= np.abs(want) * (HALF[DT[dtype]] + U32)).all()
        if scale == 1.0:
            plain = torch.empty_like(out)
            zb.z2z_embed_lookup(cb, gpu(codes), gpu(seq), W, E, plain)
            assert torch.equal(plain, out)
    st, _ = zb.z2z_status(cb)
    assert [bool(x & zb.ST_BAD_TOKEN) for x in st.tolist()] == [b in bad for b in range(B)]


def test_lookup_scaled_one_row_per_sequence_and_without_hypertokens():
    V, d, B = 50, 24, 5
    cb = session(V, d, 4, B, "bf16", [4, 3, 2, 1, 0])
    W = torch.randn(V, d, device=DEV).bfloat16()
    E = torch.randn(B, 4, d, device=DEV).bfloat16()
    codes = torch.tensor([V + 3, V + 3, 7, V, -1], dtype=torch.int32, device=DEV)     # the second has no entry 3
    out = torch.empty(B, d, dtype=torch.bfloat16, device=DEV)
    zb.z2z_embed_lookup_scaled(cb, codes, None, W, E, 2.0, out)
    want = torch.stack([E[0, 3], torch.zeros_like(W[0]), W[7], E[3, 0], torch.zeros_like(W[0])]) * 2
    assert torch.equal(out, want)
    assert zb.z2z_status(cb)[0].tolist()[:4] == [zb.ST_CAP_FROZEN, zb.ST_BAD_TOKEN, 0, 0]
    none = zb.Codebook(zb.make_config(V, d, 3, 0, B, "bf16", 0, 1, 8), DEV)           # cap 0
    zb.z2z_embed_lookup_scaled(none, torch.tensor([0, 1, 2, 49, -1], dtype=torch.int32, device=DEV), None, W, None, 0.5, out)
    assert torch.equal(out, torch.cat([W[[0, 1, 2, 49]] * 0.5, torch.zeros_like(W[:1])]))


def check_grad(cb, codes, seq, g, n, V, cap, B, scale, gdt, accumulate, base=True, hyper=True, rng=None):
    d = g.shape[1]
    old_W = torch.randn(V, d, device=DEV).to(gdt)
    old_E = torch.randn(B, cap, d, device=DEV).to(gdt)
    gW, gE = old_W.clone(), old_E.clone()
    scratch = torch.full((zb.z2z_embed_grad_scratch_bytes(cb.cfg, len(codes)),), 0xab, dtype=torch.uint8, device=DEV)
    args = (cb, gpu(codes), None if seq is None else gpu(seq), g, scale, accumulate, gW if base else None, gE if hyper else None, scratch)
    zb.z2z_embed_grad(*args)
    ok = np.ones(len(codes), bool) if seq is None else (seq >= 0) & (seq < B)
    dW, dE, cW, cE, aW, aE = oemb.lookup_grad(np.where(ok, codes, -1), None if seq is None else np.where(ok, seq, 0), f64(g), V, cap, B, n,
                                              float(np.float32(scale)))
    there = np.arange(cap)[None, :] < np.array(n)[:, None]
    for got, old, d_, c_, a_, on, own_rows in ((gW, old_W, dW, cW, aW, base, np.ones(V, bool)), (gE, old_E, dE, cE, aE, hyper, there)):
        got, old = f64(got), f64(old)
        if not on:
            assert np.array_equal(got, old)
            continue
        want = d_ + (old if accumulate else 0.0)
        err = (c_[..., None] + 4) * U32 * (a_ + (np.abs(old) if accumulate else 0.0)) + HALF[gdt] * np.abs(want)
        untouched = (c_ == 0) if accumulate else ~own_rows
        want = np.where(untouched[..., None], old, want)
        err = np.where(untouched[..., None], 0.0, err)                                 # not even rewritten
        assert (np.abs(got - want) <= err).all(), np.abs(got - want).max()
    first = (gW.clone(), gE.clone())                                                   # the same call: the same bits
    gW.copy_(old_W); gE.copy_(old_E)
    scratch.fill_(0x5c)
    zb.z2z_embed_grad(*args)
    assert torch.equal(gW, first[0]) and torch.equal(gE, first[1])


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("gdt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,d", [(1, 8), (7, 40), (100, 264), (333, 1000), (2100, 136), (5000, 48)])
def test_grad(N, d, dtype, gdt, accumulate):
    rng = np.random.default_rng(N)
    V, cap, B = 400, 33, 5
    n = [33, 0, 12, 1, 25]
    cb = session(V, d, cap, B, dtype, n)
    codes, seq = stream(rng, N, V, B, n)
    if N > 50:
        codes[10], codes[11], codes[12] = V + n[seq[10]], -9, 1 << 30
        seq[20], seq[21] = -1, B
    g = torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)).to(DT[dtype]).to(DEV)
    check_grad(cb, codes, seq, g, n, V, cap, B, 31.625, gdt, accumulate)
    st = zb.z2z_status(cb)[0].tolist()
    assert any(x & zb.ST_BAD_TOKEN for x in st) == (N > 50)


@pytest.mark.parametrize("few,share", [(1, 0.0), (2, 0.0), (3, 0.5), (40, 1.0)])
@pytest.mark.parametrize("N", [63, 64, 65, 1023, 1025, 4097, 9001])
def test_grad_of_few_targets(N, few, share):
    # long runs of one target, that begin and end anywhere
    rng = np.random.default_rng(N + few)
    V, cap, B, d = 64, 4, 2, 72
    n = [4, 1]
    cb = session(V, d, cap, B, "bf16", n)
    codes, seq = stream(rng, N, V, B, n, share, few)
    g = torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)).bfloat16().to(DEV)
    check_grad(cb, codes, seq, g, n, V, cap, B, 1.0, torch.float32, False)
    check_grad(cb, codes, seq, g, n, V, cap, B, -2.0, torch.bfloat16, True)


@pytest.mark.parametrize("base,hyper", [(True, False), (False, True)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_grad_of_one_table(base, hyper, accumulate):
    rng = np.random.default_rng(3)
    V, cap, B, d, N = 100, 9, 3, 64, 700
    n = [9, 4, 0]
    cb = session(V, d, cap, B, "bf16", n)
    codes, seq = stream(rng, N, V, B, n)
    g = torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)).bfloat16().to(DEV)
    check_grad(cb, codes, seq, g, n, V, cap, B, 8.0, torch.float32, accumulate, base, hyper)


def test_grad_without_rows_and_without_tokens():
    V, cap, B, d = 30, 5, 2, 16
    n = [3, 5]
    cb = session(V, d, cap, B, "fp32", n)
    for codes in (np.zeros(0, np.int32), np.full(9, -1, np.int32)):
        seq = np.zeros(len(codes), np.int32)
        g = torch.randn(len(codes), d, device=DEV)
        for accumulate in (False, True):
            check_grad(cb, codes, seq, g, n, V, cap, B, 1.0, torch.float32, accumulate)
    check_grad(cb, np.array([V + 2, 29], np.int32), None, torch.randn(2, d, device=DEV), n, V, cap, B, 3.0, torch.float32, True)
    assert zb.z2z_status(cb)[0].tolist() == [0, zb.ST_CAP_FROZEN]


def test_grad_keeps_infinities_and_nan_to_their_rows():
    V, cap, B, d, N = 40, 4, 1, 32, 300
    cb = session(V, d, cap, B, "fp32", [4])
    rng = np.random.default_rng(8)
    codes = rng.integers(0, V, N).astype(np.int32)
    codes[5], codes[6], codes[7] = 3, 3, -1
    g = torch.randn(N, d, device=DEV)
    g[5, 0], g[6, 1], g[7] = float("inf"), float("nan"), float("nan")          # row 7 has no token: not taken
    gW = torch.zeros(V, d, device=DEV)
    scratch = torch.empty(zb.z2z_embed_grad_scratch_bytes(cb.cfg, N), dtype=torch.uint8, device=DEV)
    zb.z2z_embed_grad(cb, gpu(codes), torch.zeros(N, dtype=torch.int32, device=DEV), g, 2.0, False, gW, None, scratch)
    bad = ~torch.isfinite(gW)
    assert bad.sum().item() == 2 and gW[3, 0].item() == float("inf") and torch.isnan(gW[3, 1]).item()


@pytest.mark.parametrize("N", [900, 30000])
def test_grad_replayed_from_a_graph_on_another_stream(N):
    rng = np.random.default_rng(4)
    V, cap, B, d = 200, 16, 4, 128
    n = [16, 5, 9, 0]
    cb = session(V, d, cap, B, "bf16", n)
    codes, seq = stream(rng, N, V, B, n)
    gc, gs = gpu(codes), gpu(seq)
    g = torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)).bfloat16().to(DEV)
    gW, gE = torch.zeros(V, d, device=DEV), torch.zeros(B, cap, d, device=DEV)
    scratch = torch.empty(zb.z2z_embed_grad_scratch_bytes(cb.cfg, N), dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        zb.z2z_embed_grad(cb, gc, gs, g, 1.0, False, gW, gE, scratch)
    for k in range(3):                                       # other inputs in the same buffers
        codes, seq = stream(rng, N, V, B, n, few=1 + 60 * k)
        gc.copy_(gpu(codes)); gs.copy_(gpu(seq)); g.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        dW, dE, cW, cE, aW, aE = oemb.lookup_grad(codes, seq, f64(g), V, cap, B, n, 1.0)
        assert (np.abs(f64(gW) - dW) <= (cW[:, None] + 4) * U32 * aW + U32 * np.abs(dW)).all()
        assert (np.abs(f64(gE) - dE) <= (cE[..., None] + 4) * U32 * aE + U32 * np.abs(dE)).all()


@pytest.mark.parametrize("N", [20011, 70003])
def test_grad_of_a_large_batch(N):
    # every path of the sort, a vocabulary beyond 16 bits, rows sampled against sums in 64 bits
    rng = np.random.default_rng(N)
    V, cap, B, d = 90001, 500, 7, 40
    n = [500, 0, 123, 499, 1, 300, 250]
    cb = session(V, d, cap, B, "bf16", n)
    seq = np.sort(rng.integers(0, B, N)).astype(np.int32)
    codes = np.minimum(np.exp(rng.random(N) * np.log(V)), V - 1).astype(np.int32)          # Zipf: a few long runs
    hyp = rng.random(N) < 0.4
    nn = np.array(n)[seq]
    codes = np.where(hyp & (nn > 0), V + (rng.random(N) * nn).astype(np.int32), codes).astype(np.int32)
    g = torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)).bfloat16().to(DEV)
    check_grad(cb, codes, seq, g, n, V, cap, B, 2.0, torch.float32, False)
    check_grad(cb, codes, seq, g, n, V, cap, B, 2.0, torch.float32, True)


@pytest.mark.parametrize("N,V,cap,d", [(3000, 300000, 10, 8), (160001, 1000, 65535, 8), (310001, 200000, 700, 24)])
def test_grad_of_many_targets_and_rows(N, V, cap, d):
    # targets beyond 18 bits (three passes of the sort), more rows than a block's registers hold, long chunks
    rng = np.random.default_rng(N)
    B = 5
    n = [min(cap, V - 2), 0, min(cap, 700) // 2, min(cap, 1), min(cap, 500)]
    cb = session(V, d, cap, B, "bf16", [min(x, V - 2) for x in n])
    seq = np.sort(rng.integers(0, B, N)).astype(np.int32)
    nn = np.array(n)[seq]
    codes = np.minimum(np.exp(rng.random(N) * np.log(V)), V - 1).astype(np.int64)
    codes = np.where((rng.random(N) < 0.5) & (nn > 0), V + (rng.random(N) * nn).astype(np.int64), codes)
    codes[rng.random(N) < 0.02] = -1
    codes = codes.astype(np.int32)
    g = torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)).bfloat16().to(DEV)
    check_grad(cb, codes, seq, g, n, V, cap, B, 2.0, torch.float32, False)
    check_grad(cb, codes, seq, g, n, V, cap, B, 0.5, torch.bfloat16, True)


@pytest.mark.parametrize("N,V,cap,d", [(723, 500, 10, 4096), (725, 500, 10, 4096), (1000, 500, 10, 4096), (1000, 140000, 3, 8), (1000, 300000, 0, 8),
                                       (300, 2000000, 2, 8), (129, 500, 10, 16384)])
def test_grad_of_few_rows_with_many_columns_or_targets(N, V, cap, d):
    test_grad_of_many_targets_and_rows(N, V, cap, d)


def test_grad_on_two_streams_with_scratch_of_their_own():
    rng = np.random.default_rng(31)
    V, cap, B, d = 500, 20, 3, 256
    n = [20, 7, 0]
    jobs = []
    for N in (700, 20000):
        cb = session(V, d, cap, B, "bf16", n)
        codes, seq = stream(rng, N, V, B, n)
        g = torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)).bfloat16().to(DEV)
        gW, gE = torch.zeros(V, d, device=DEV), torch.zeros(B, cap, d, device=DEV)
        scratch = torch.empty(zb.z2z_embed_grad_scratch_bytes(cb.cfg, N), dtype=torch.uint8, device=DEV)
        jobs.append((cb, gpu(codes), gpu(seq), g, 1.0, False, gW, gE, scratch))
    want = []
    for j in jobs:
        zb.z2z_embed_grad(*j)
        want.append((j[6].clone(), j[7].clone()))
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, j in zip(streams, jobs):
            with torch.cuda.stream(s):
                j[6].fill_(3.0)
                zb.z2z_embed_grad(*j)
        torch.cuda.synchronize()
        for j, (a, b) in zip(jobs, want):
            assert torch.equal(j[6], a) and torch.equal(j[7], b)
