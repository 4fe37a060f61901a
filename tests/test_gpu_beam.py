"""Beam selection and reordering against the oracle: codes, parents, flags and copies are exact, a score is the fp64
sum rounded once to fp32."""
import numpy as np
import pytest
import torch

from oracle import beam as obeam
from paper_2506_01084_b200 import binding as zb
from tests.test_gpu_embed_scaled import session

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def run_select(cb, beams, l32, n, lse, scores, fin, eos, alias=False, flags=True):
    B = l32.shape[0]
    V = cb.cfg.V
    g = torch.from_numpy(l32).to(DEV)
    sc = torch.from_numpy(scores).to(DEV)
    fi = None if fin is None else torch.from_numpy(fin).to(DEV)
    parent, code = torch.full((2, B), -77, dtype=torch.int32, device=DEV).unbind(0)
    ns = sc if alias else torch.full((B,), 3.0, device=DEV)
    nf = (fi if alias and fi is not None else torch.full((B,), 9, dtype=torch.uint8, device=DEV)) if flags else None
    act = torch.full((B,), 9, dtype=torch.uint8, device=DEV) if flags else None
    zb.z2z_beam_select(cb, beams, g, torch.from_numpy(lse).to(DEV), sc, fi, eos, parent, code, ns, nf, act)
    want = obeam.select(beams, [l32[b, :V + n[b]] for b in range(B)], lse, scores, fin, eos)
    assert parent.tolist() == want[0]
    assert code.tolist() == want[1]
    assert np.array_equal(ns.cpu().numpy(), np.array(want[2]).astype(np.float32))
    if flags:
        assert nf.tolist() == want[3] and act.tolist() == want[4]
    return want


def inputs(rng, B, V, cap, n, spread=2.0):
    l = (rng.standard_normal((B, V + cap)) * spread).astype(np.float32)
    lse = np.array([np.log(np.exp(l[b, :V + n[b]].astype(np.float64)).sum()) for b in range(B)], dtype=np.float32)
    for b in range(B):
        l[b, V + n[b]:] = 60.0                               # behind a row's columns: never taken
    scores = (-10 + rng.standard_normal(B)).astype(np.float32)
    return l, lse, scores


@pytest.mark.parametrize("beams", [1, 2, 3, 5, 8, 17, 32])
@pytest.mark.parametrize("V,cap", [(40, 7), (999, 30), (32064, 100), (50021, 0)])
def test_beam_select(beams, V, cap):
    rng = np.random.default_rng(V + beams)
    G = 3 if V < 40000 else 2
    B = G * beams
    n = [int(x) for x in rng.integers(0, cap + 1, B)] if cap else [0] * B
    cb = session(V, 8, cap, B, "fp32", n)
    for k in range(4):
        l, lse, scores = inputs(rng, B, V, cap, n)
        fin = None
        if k == 1:                                           # a request's first step: one beam is alive
            for g in range(G):
                scores[g * beams + 1:(g + 1) * beams] = -np.inf
        if k >= 2:
            fin = (rng.random(B) < 0.3).astype(np.uint8)
            scores[rng.random(B) < 0.2] = -np.inf
        eos = int(np.argmax(l[0, :V])) if k != 3 else -1
        run_select(cb, beams, l, n, lse, scores, fin, eos, alias=k == 2, flags=k != 1)


@pytest.mark.parametrize("beams", [2, 7, 32])
def test_beam_select_ties_take_the_lower_beam_and_column(beams):
    rng = np.random.default_rng(beams)
    V, cap = 5003, 20
    B = 2 * beams
    n = [(3 * b) % 21 for b in range(B)]
    cb = session(V, 8, cap, B, "fp32", n)
    for k in range(6):
        l = rng.integers(-3, 2 if k % 2 else 1, (B, V + cap)).astype(np.float32) * np.float32(0.5)
        l[l == 0] *= np.where(rng.random((l == 0).sum()) < 0.5, -1, 1).astype(np.float32)          # +0 and -0 are equal
        scores = rng.integers(-2, 1, B).astype(np.float32)
        run_select(cb, beams, l, n, np.full(B, 2.0, np.float32), scores, (rng.random(B) < 0.2).astype(np.uint8), 3)
    l = np.zeros((B, V + cap), np.float32)                   # all equal
    run_select(cb, beams, l, n, np.full(B, 8.0, np.float32), np.zeros(B, np.float32), None, -1)
    l = np.tile(np.arange(V + cap, dtype=np.float32), (B, 1))                  # every column better than the one before
    run_select(cb, beams, l, n, np.full(B, 8.0, np.float32), np.zeros(B, np.float32), None, -1)
    run_select(cb, beams, -l, n, np.full(B, 8.0, np.float32), np.zeros(B, np.float32), None, -1)


def test_beam_select_of_masked_infinite_and_missing_values():
    rng = np.random.default_rng(9)
    V, cap, beams = 700, 10, 4
    B = 6 * beams
    n = [b % 11 for b in range(B)]
    cb = session(V, 8, cap, B, "fp32", n)
    l, lse, scores = inputs(rng, B, V, cap, n)
    l[0:4] = -np.inf                                         # nothing visible at all: the group dies
    l[4] = -np.inf
    l[4, 5] = 1.0                                            # one column left
    l[5:8] = np.float32(np.finfo(np.float32).min)            # masked with the type's lowest value: still candidates
    l[8, 100:300] = np.nan                                   # NaN is no candidate
    l[9] = np.nan
    l[12, 17] = np.inf                                       # an overflowed logit wins
    lse[13] = np.nan
    scores[16:20] = -np.inf                                  # a dead group
    scores[20], scores[21] = np.nan, np.inf
    run_select(cb, beams, l, n, lse, scores, None, -1)
    fin = np.zeros(B, np.uint8)
    fin[[9, 16, 20]] = 1                                     # a finished beam's logits are not looked at
    run_select(cb, beams, l, n, lse, scores, fin, 4)


@pytest.mark.parametrize("V", [1, 2, 3, 7])
@pytest.mark.parametrize("beams", [1, 5, 32])
def test_beam_select_with_fewer_columns_than_beams(V, beams):
    rng = np.random.default_rng(V)
    B = 4 * beams
    cb = session(V, 8, 0, B, "fp32", [0] * B)
    for k in range(4):
        l, lse, scores = inputs(rng, B, V, 0, [0] * B)
        scores[rng.random(B) < 0.7] = -np.inf                # a few candidates at most: dead slots
        run_select(cb, beams, l, [0] * B, lse, scores, (rng.random(B) < 0.3).astype(np.uint8) if k else None, 0 if k == 2 else -1)


@pytest.mark.parametrize("beams", [3, 32])
def test_beam_select_when_one_thread_has_the_best_columns(beams):
    # the best columns 1024 apart: those of one vector of one thread in every tile, far more than the list takes
    V, cap = 70001, 3
    rng = np.random.default_rng(beams)
    cb = session(V, 8, cap, beams, "fp32", [2] * beams)
    l, lse, scores = inputs(rng, beams, V, cap, [2] * beams)
    for b in range(beams):
        for k in range(4):
            at = np.arange((5 * b) % 1000 + k, V, 1024)
            l[b, at] = 30 + rng.integers(0, 3, at.size)      # ties among them
    run_select(cb, beams, l, [2] * beams, lse, scores, None, -1)


def test_beam_select_of_many_beams():
    rng = np.random.default_rng(77)
    V, cap, beams = 3001, 9, 4
    B = 1024
    n = [b % 10 for b in range(B)]
    cb = session(V, 8, cap, B, "fp32", n)
    l, lse, scores = inputs(rng, B, V, cap, n)
    run_select(cb, beams, l, n, lse, scores, (rng.random(B) < 0.2).astype(np.uint8), 3)
    parent = torch.arange(B, dtype=torch.int32)
    parent[1::2] = parent[0::2]
    hist = torch.arange(B, dtype=torch.int32, device=DEV).view(B, 1).clone()
    E = torch.arange(B, device=DEV).view(B, 1, 1).expand(B, cap, 8).float().contiguous()
    zb.z2z_beam_reorder(cb, parent.to(DEV), E, E, states=(hist,))
    nn = zb.z2z_status(cb)[1].tolist()
    assert nn == [n[p] for p in parent.tolist()] and hist.view(-1).tolist() == parent.tolist()
    for b in (0, 1, 2, 511, 512, 1023):
        assert (E[b, :nn[b]] == int(parent[b])).all() and (E[b, nn[b]:] == b).all()


def test_beam_select_scores_in_64_bits():
    # sums that fp32 would round to the same value, or in another order
    V, cap, beams = 64, 0, 4
    cb = session(V, 8, cap, beams, "fp32", [0] * beams)
    l = np.full((beams, V), -50.0, np.float32)
    scores = np.array([-1e6, -1e6, -1e6, -1e6], np.float32)
    lse = np.array([1.0, 1.0, 1.0, 1.0], np.float32)
    l[0, 3], l[1, 2], l[2, 9], l[3, 1] = 0.001, 0.004, 0.002, 0.003
    want = run_select(cb, beams, l, [0] * beams, lse, scores, None, -1)
    assert want[0] == [0, 1, 2, 3]
    l[0, 4], l[1, 7] = 0.0035, 0.0041
    run_select(cb, beams, l, [0] * beams, lse, scores, None, -1)


def book(cb, b):
    cons, ln = zb.z2z_codebook_read(cb, b)
    return cons, ln


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,cap", [(8, 5), (72, 130), (1000, 64)])
def test_beam_reorder(dtype, d, cap):
    rng = np.random.default_rng(d + cap)
    V, W, G = 400, 4, 5
    B = W * G
    n = [int(x) for x in rng.integers(0, cap + 1, B)]
    n[0], n[1], n[2] = cap, 0, 1
    cb = session(V, d, cap, B, dtype, n)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    E, U = (torch.randn(B, cap, d, device=DEV).to(dt) for _ in range(2))
    Ef, Uf = (torch.randn(B, cap, d, device=DEV) for _ in range(2))
    hist = torch.randint(0, 9999, (B, 37), dtype=torch.int32, device=DEV)
    wide = torch.randn(B, 50, device=DEV)
    view = wide[:, 3:21]                                     # rows apart, not 16-byte aligned
    kv = torch.randn(B, 2, 3, 8, device=DEV).bfloat16()
    parent = np.arange(B, dtype=np.int32)
    parent[1], parent[2], parent[3] = 0, 0, 0                # all from one: longer and shorter codebooks are overwritten
    parent[4], parent[7] = 5, 6
    parent[8:12] = [9, 9, 9, 11]
    parent[12:16] = [12, 13, 14, 15]                         # nothing moves
    parent[16] = 19
    before = [t.clone() for t in (E, U, Ef, Uf, hist, wide, kv)]
    books = [book(cb, b) for b in range(B)]
    st0, n0 = zb.z2z_status(cb)
    zb.z2z_beam_reorder(cb, torch.from_numpy(parent).to(DEV), E, U, Ef, Uf, (hist, view, kv))
    st, nn = zb.z2z_status(cb)
    for b in range(B):
        p = int(parent[b])
        assert nn[b] == n0[p] and st[b] == st0[p]
        cons, ln = book(cb, b)
        assert torch.equal(cons, books[p][0]) and torch.equal(ln, books[p][1])
        k = n[p] if p != b else 0
        for now, old in zip((E, U, Ef, Uf), before):
            assert torch.equal(now[b, :k], old[p, :k]) and torch.equal(now[b, k:], old[b, k:])
        assert torch.equal(hist[b], before[4][p]) and torch.equal(kv[b], before[6][p])
        assert torch.equal(wide[b, 3:21], before[5][p, 3:21])
        assert torch.equal(wide[b, :3], before[5][b, :3]) and torch.equal(wide[b, 21:], before[5][b, 21:])
    # the hash came along: what a sequence does next is what its parent does
    tok = torch.randint(0, 60, (B, 30), dtype=torch.int32, device=DEV)
    par = torch.from_numpy(parent).to(DEV).long()
    tok = tok[par].contiguous()
    codes, lens = torch.zeros_like(tok), torch.zeros(B, dtype=torch.int32, device=DEV)
    for t in range(30):
        zb.z2z_lzw_step(cb, tok[:, t].contiguous(), None, None)
    st, nn = zb.z2z_status(cb)
    for b in range(B):
        p = int(parent[b])
        assert nn[b] == nn[p]
        assert all(torch.equal(x, y) for x, y in zip(book(cb, b), book(cb, p)))
    zb.z2z_lzw_encode(cb, tok, None, codes, lens)            # and parses with it
    assert torch.equal(codes, codes[par]) and torch.equal(lens, lens[par])


def test_beam_reorder_refuses_parents_that_are_overwritten():
    V, d, cap, B = 100, 8, 10, 6
    n = [10, 3, 4, 5, 6, 7]
    cb = session(V, d, cap, B, "fp32", n)
    E, U = torch.randn(B, cap, d, device=DEV), torch.randn(B, cap, d, device=DEV)
    e0, u0 = E.clone(), U.clone()
    parent = torch.tensor([1, 0, 3, 3, 6, -1], dtype=torch.int32, device=DEV)         # a swap, one that is right, two out of range
    hist = torch.arange(B, dtype=torch.int32, device=DEV).view(B, 1).clone()
    zb.z2z_beam_reorder(cb, parent, E, U, states=(hist,))
    st, nn = zb.z2z_status(cb)
    bad = [bool(x & zb.ST_BAD_PARENT) for x in st.tolist()]
    assert bad == [True, True, False, False, True, True]
    assert nn.tolist() == [10, 3, 5, 5, 6, 7] and hist.view(-1).tolist() == [0, 1, 3, 3, 4, 5]
    for b in (0, 1, 3, 4, 5):
        assert torch.equal(E[b], e0[b]) and torch.equal(U[b], u0[b])
    assert torch.equal(E[2, :5], e0[3, :5]) and torch.equal(U[2, 5:], u0[2, 5:])


def test_beam_reorder_without_hypertokens_and_with_tied_tables():
    B = 3
    cb = zb.Codebook(zb.make_config(50, 8, 3, 0, B, "fp32", 0, 1, 8), DEV)
    hist = torch.arange(B * 4, dtype=torch.int32, device=DEV).view(B, 4).clone()
    parent = torch.tensor([0, 0, 2], dtype=torch.int32, device=DEV)
    zb.z2z_beam_reorder(cb, parent, None, None, states=(hist,))
    assert hist[1].tolist() == [0, 1, 2, 3] and hist[2].tolist() == [8, 9, 10, 11]
    zb.z2z_beam_reorder(cb, parent, None, None)
    cb = session(50, 16, 6, B, "bf16", [6, 2, 4])
    E = torch.randn(B, 6, 16, device=DEV).bfloat16()
    e0 = E.clone()
    zb.z2z_beam_reorder(cb, parent, E, E)
    assert torch.equal(E[1], e0[0]) and torch.equal(E[0], e0[0]) and torch.equal(E[2], e0[2])


def test_beam_reorder_of_a_large_session():
    # many sequences, offsets beyond 32 bits in the caches
    V, d, cap, B = 5000, 2048, 1024, 520
    n = [(b * 37) % 900 for b in range(B)]
    cb = session(V, d, cap, B, "bf16", n)
    E = torch.empty(B, cap, d, dtype=torch.bfloat16, device=DEV)
    for b in range(B):
        E[b] = b % 251
    E[:, :, 0] = torch.arange(cap, device=DEV) % 249
    parent = torch.arange(B, dtype=torch.int32)
    parent[1::4], parent[515] = parent[0::4], 519
    zb.z2z_beam_reorder(cb, parent.to(DEV), E, E)
    st, nn = zb.z2z_status(cb)
    assert nn.tolist() == [n[p] for p in parent.tolist()]
    for b in (0, 1, 2, 3, 257, 513, 515, 516, 517, 519):
        p = int(parent[b])
        k = n[p]
        assert (E[b, :k, 1:] == p % 251).all() and (E[b, k:, 1:] == b % 251).all()
        assert torch.equal(E[b, :, 0], (torch.arange(cap, device=DEV) % 249).bfloat16())


def test_beam_calls_replayed_from_a_graph():
    rng = np.random.default_rng(2)
    V, cap, beams, d = 3001, 40, 4, 64
    B = 2 * beams
    n = [5 * b for b in range(B)]
    cb = session(V, d, cap, B, "bf16", n)
    E, U = torch.zeros(2, B, cap, d, dtype=torch.bfloat16, device=DEV).unbind(0)
    l, lse, scores = inputs(rng, B, V, cap, n)
    gl, ge, gs = torch.from_numpy(l).to(DEV), torch.from_numpy(lse).to(DEV), torch.from_numpy(scores).to(DEV)
    fin = torch.zeros(B, dtype=torch.uint8, device=DEV)
    parent, code = torch.empty(2, B, dtype=torch.int32, device=DEV).unbind(0)
    act = torch.empty(B, dtype=torch.uint8, device=DEV)
    hist = torch.zeros(B, 2, dtype=torch.int32, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        zb.z2z_beam_select(cb, beams, gl, ge, gs, fin, 7, parent, code, gs, fin, act)
        zb.z2z_beam_reorder(cb, parent, E, U, states=(hist,))
    books = n
    for k in range(4):
        l, lse, _ = inputs(rng, B, V, cap, books)
        gl.copy_(torch.from_numpy(l)); ge.copy_(torch.from_numpy(lse))
        E.copy_(torch.arange(B, device=DEV).view(B, 1, 1).expand_as(E)); U.copy_(-E)
        hist.copy_(torch.arange(B, device=DEV).view(B, 1).expand(B, 2))
        old_s, old_f = gs.cpu().numpy(), fin.cpu().numpy()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = obeam.select(beams, [l[b, :V + books[b]] for b in range(B)], lse, old_s, old_f, 7)
        assert parent.tolist() == want[0] and code.tolist() == want[1] and fin.tolist() == want[3] and act.tolist() == want[4]
        assert np.array_equal(gs.cpu().numpy(), np.array(want[2]).astype(np.float32))
        st, nn = zb.z2z_status(cb)
        assert nn.tolist() == [books[p] for p in want[0]]
        books = nn.tolist()
        assert hist[:, 0].tolist() == want[0]
        for b in range(B):
            p = want[0][b]
            assert (E[b, :books[b]] == p).all() and (U[b, :books[b]] == -p).all() and (E[b, books[b]:] == b).all()
