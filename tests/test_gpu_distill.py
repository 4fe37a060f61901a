"""Distillation of joint logits from a teacher's top logits against the fp64 oracle.

Bounds, with u = 2^-24 and a row of C columns.  An exponential's argument (l - m) / T is off by 5 u of its size (the
difference, three roundings in the factor 1 / T log2 e, the product) and the exponential by 4 u more.  In the
normaliser s the error of an argument counts with its own probability, and the mean size of an argument under q is at
most ln C; the sum itself adds one u per addition of a chain, and a chain is one thread's or one level of a tree: at
most C / 256 + 32.  So s has the relative error e_s = (5 ln C + C / 256 + 40) u, lse = m / T + log s that plus 2 u of its
parts.  A gradient k (q - p) has q off by (6 |x| + 16) u + e_s of itself with x = (|l| + |m|) / T + |lse|, p alike over the
teacher's K entries, 3 u for the products, and one rounding to its type.  A term of the loss has the error of its
bracket log p - log q (as lse, for both) plus p's."""
import numpy as np
import pytest
import torch

from oracle import distill as odis
from paper_2506_01084_b200 import binding as zb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
u = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def f64(t):
    return t.detach().cpu().double().numpy()


def bounds(l, ids, t, T, w, dt, want_grad):
    """Error bounds of loss, lse and the (weighted) gradient of one row."""
    C = l.size
    fin = l[l > -np.inf]
    m = fin.max()
    x = (l - m) / T
    s = np.exp(x).sum()
    lse = m / T + np.log(s)
    e_s = (5 * np.log(C + 1) + C / 256 + 40) * u
    b_lse = e_s + 2 * u * (abs(m / T) + abs(np.log(s)) + abs(lse))
    keep = (ids >= 0) & (ids < C) & (t > -np.inf)
    K = max(1, keep.sum())
    ids, t = ids[keep], t[keep]
    if ids.size == 0:
        return 0.0, b_lse, np.zeros(C)
    y = (t - t.max()) / T
    ts = np.exp(y).sum()
    p = np.exp(y) / ts
    e_t = (5 * np.log(K + 1) + K + 40) * u
    e_p = (6 * np.abs(y) + 16) * u + e_t
    bracket = y - np.log(ts) - (x[ids] - np.log(s))
    with np.errstate(invalid="ignore"):
        b_br = 6 * u * (np.abs(y) + np.abs(x[ids])) + 3 * u * (np.log(ts) + np.log(s)) + e_s + e_t + 4 * u * np.abs(bracket)
        b_loss = T * T * (np.where(p > 0, p * (b_br + e_p * np.abs(bracket)), 0)).sum() * 1.01 + (K + 8) * u * T * T * np.abs(np.where(p > 0, p * bracket, 0)).sum()
    q = np.exp(x) / s
    with np.errstate(invalid="ignore"):
        # (fp32 underflow: what is smaller than 2^-126 may be 0)
        b_q = np.where(q > 0, q * (6 * u * ((np.abs(l) + abs(m)) / T + abs(lse)) + 16 * u + e_s + b_lse), 0) + 2.0 ** -126
    b_p = np.zeros(C)
    np.add.at(b_p, ids, p * (e_p + K * u))
    k = abs(w) * T
    return b_loss, b_lse, k * (b_q + b_p) * 1.01 + 3 * u * np.abs(want_grad) + HALF[dt] * np.abs(want_grad) + k * 2.0 ** -126


def check(logits, n_cols, ids, t, T, w, ld=None, in_place=False, rows=None):
    """All forms of the call on one batch, held against the oracle row by row (`rows`: in these).  logits: fp32 / bf16 host
    tensor [N, cols]."""
    N, cols = logits.shape
    dt = logits.dtype
    ld = ld or cols
    buf = torch.full((N, ld), 777.0, dtype=dt, device=DEV)
    g_l = buf[:, :cols]
    g_l.copy_(logits)
    gn = None if n_cols is None else torch.tensor(n_cols, dtype=torch.int32, device=DEV)
    gi = None if ids is None else torch.from_numpy(ids.astype(np.int32)).to(DEV)
    gt = None if t is None else torch.from_numpy(t.astype(np.float32)).to(DEV)
    gw = None if w is None else torch.from_numpy(w.astype(np.float32)).to(DEV)
    loss, lse = torch.full((2, N), 55.0, device=DEV).unbind(0)
    zb.z2z_distill_loss(g_l, gn, gi, gt, T, None, loss, lse)
    g1 = torch.full((N, ld), 9.0, dtype=dt, device=DEV)
    loss2, lse2 = torch.full((2, N), 55.0, device=DEV).unbind(0)
    zb.z2z_distill_loss(g_l, gn, gi, gt, T, gw, loss2, lse2, g1[:, :cols])
    g2 = torch.full((N, ld), 9.0, dtype=dt, device=DEV)
    ones = torch.ones(N, device=DEV) if gw is None else gw
    zb.z2z_distill_grad(g_l, gn, gi, gt, T, lse, ones, g2[:, :cols])
    for g in (g1, g2):
        assert (g[:, cols:] == 9.0).all()                    # what lies between the rows is not touched
    assert (buf[:, cols:] == 777.0).all()
    L = f64(logits)
    for r in range(N) if rows is None else rows:
        C = cols if n_cols is None else min(max(int(n_cols[r]), 0), cols)
        l = L[r, :C]
        ii = np.zeros(0, np.int64) if ids is None else ids[r].astype(np.int64)
        tt = np.zeros(0) if t is None else t[r].astype(np.float32).astype(np.float64)
        wr = 1.0 if w is None else float(np.float32(w[r]))
        has = ((ii >= 0) & (ii < C) & (tt > -np.inf)).any()
        if np.isnan(l).any() or (l == np.inf).any():
            assert torch.isnan(lse[r]) and torch.isnan(lse2[r])
            for g in (g1, g2):
                if has and wr != 0:
                    assert torch.isnan(g[r, :C]).all() and torch.isnan(loss[r])
                else:
                    assert (g[r, :C] == 0).all()
                assert (g[r, C:cols] == 0).all()
            continue
        want_loss, want_lse, want = odis.row(l, ii, tt, T) if C else (0.0, -np.inf, np.zeros(0))
        if C == 0 or l.max() <= -2.0 ** 126:
            for v in (loss, loss2):
                assert v[r].item() == 0.0
            for v in (lse, lse2):
                assert v[r].item() == -np.inf
            assert (g1[r, :cols] == 0).all() and (g2[r, :cols] == 0).all()
            continue
        want = want * wr
        b_loss, b_lse, b_g = bounds(l, ii, tt, T, wr, dt, want)
        for a, b in ((loss, lse), (loss2, lse2)):
            assert abs(b[r].item() - want_lse) <= b_lse, (r, b[r].item(), want_lse, b_lse)
            if np.isinf(want_loss):
                assert a[r].item() == want_loss
            else:
                assert abs(a[r].item() - want_loss) <= b_loss + 1e-30, (r, a[r].item(), want_loss, b_loss)
        if not has or wr == 0:
            want, b_g = np.zeros(C), np.zeros(C)
        for g in (g1, g2):
            err = np.abs(f64(g[r, :C]) - want)
            assert (err <= b_g).all(), (r, err.max(), (err / np.maximum(b_g, 1e-300)).max(), int(np.argmax(err / np.maximum(b_g, 1e-300))))
            assert (g[r, C:cols] == 0).all()
    if in_place:
        for kind in (0, 1):
            same = buf.clone()
            if kind == 0:
                zb.z2z_distill_loss(same[:, :cols], gn, gi, gt, T, gw, loss2, lse2, same[:, :cols])
            else:
                zb.z2z_distill_grad(same[:, :cols], gn, gi, gt, T, lse, ones, same[:, :cols])
            want = (g1, g2)[kind]
            assert torch.equal(same[:, :cols].isnan(), want[:, :cols].isnan())
            assert torch.equal(same[:, :cols].nan_to_num(), want[:, :cols].nan_to_num())
            assert (same[:, cols:] == 777.0).all()


def batch(rng, N, cols, K, dt, spread=2.0, exact_cols=False):
    l = rng.standard_normal((N, cols)).astype(np.float32) * spread
    ids = np.stack([rng.choice(cols, K, replace=K > cols) for _ in range(N)]) if K else None
    t = (rng.standard_normal((N, K)) * 2 + 5).astype(np.float32) if K else None
    if K:
        for r in range(N):
            l[r, ids[r]] += t[r] * 0.7
        ids[rng.random((N, K)) < 0.1] = -1
    n_cols = None if exact_cols else [max(1, cols - int(x)) for x in rng.integers(0, max(cols // 3, 1), N)]
    return torch.from_numpy(l).to(dt), n_cols, ids, t


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("N,cols,K", [(1, 1, 1), (3, 7, 5), (5, 64, 1), (4, 1000, 50), (2, 4099, 128), (3, 33001, 64), (2, 40960, 1024)])
def test_distill(dt, T, N, cols, K):
    rng = np.random.default_rng(cols + K)
    l, n, ids, t = batch(rng, N, cols, K, dt)
    w = rng.random(N).astype(np.float32) + 0.1
    check(l, n, ids, t, T, w, in_place=True)
    check(l, None, ids, t, T, None, ld=cols + 5)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [128256 + 2048, 128256 + 2053, 300007])
def test_distill_of_large_vocabularies(dt, cols):
    # rows that take several blocks' shared memory, and rows beyond what a cluster holds
    rng = np.random.default_rng(cols)
    l, n, ids, t = batch(rng, 3, cols, 64, dt)
    check(l, n, ids, t, 1.0, np.array([0.3, 1.0, 2.0]), in_place=True)
    check(l, None, ids, t, 2.0, None, ld=cols + 3)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_distill_of_a_row_too_long_to_be_held(dt):
    rng = np.random.default_rng(77)
    cols = 1000003
    l, n, ids, t = batch(rng, 2, cols, 32, dt)
    check(l, [cols, cols - 70001], ids, t, 1.0, np.array([1.0, 0.5]), in_place=True)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [5, 1003, 50021])
def test_distill_edges(dt, cols):
    """Rows without columns, masked rows, rows without a teacher, duplicates, weights of zero, infinities and NaN."""
    rng = np.random.default_rng(cols)
    N, K = 15, 5
    l, n, ids, t = batch(rng, N, cols, K, dt, exact_cols=True)
    n = [cols] * N
    n[0] = 0
    n[1] = -3
    n[2] = cols + 9
    l[3] = -np.inf
    l[4, :] = -np.inf
    l[4, 2] = 1.5                                            # one column left, the teacher may not name it
    ids[4, 0] = 2
    l[5, 1:] = torch.finfo(dt).min                           # masked with the type's lowest value
    ids[5] = [0, -1, -1, -1, -1]
    ids[6] = -1                                              # no teacher
    ids[7] = [3, 3, 1, 3, 1]                                 # the same column more than once
    t[8, 1:] = -np.inf
    t[9] = -np.inf                                           # no teacher either
    l[10, 3] = np.nan
    l[11, 0] = np.inf
    n[12] = max(1, cols // 2)
    ids[12, :3] = [n[12] - 1, n[12], cols - 1]               # the last visible column, and two that are not
    l[12, n[12]:] = np.nan                                   # nothing behind the columns is read
    l[13, 1] = np.nan
    l[14] = torch.finfo(dt).min                              # masked throughout with it: as a row of -inf
    w = np.ones(N, np.float32)
    w[13] = 0.0                                              # padding: gradient 0 whatever the row holds
    w[8] = -0.5
    check(l, n, ids, t, 1.0, w, in_place=True)
    check(l, n, ids, t, 2.5, w, ld=cols + 1)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,cols,K", [(300, 9001, 5), (301, 20483, 127), (350, 33000, 128), (297, 40001, 0), (160, 65537, 33), (80, 140000, 64), (75, 262147, 3), (200, 20001, 256),
                                      (149, 290001, 7)])
def test_distill_of_many_rows(dt, N, cols, K):
    # more rows than the blocks take at once: rows of every length, among them such without columns, without a
    # teacher, with a weight of zero and with NaN, next to ordinary ones
    rng = np.random.default_rng(N + cols)
    l = (torch.from_numpy(rng.standard_normal((N, cols)).astype(np.float32)) * 2).to(dt)
    ids = rng.integers(0, cols, (N, K)) if K else None
    t = (rng.standard_normal((N, K)) * 2 + 5).astype(np.float32) if K else None
    n = [cols - int(x) for x in rng.integers(0, cols // 2, N)]
    n[3], n[4], n[9], n[N - 1] = 0, cols, 1, 7
    w = rng.random(N).astype(np.float32) + 0.1
    w[5], w[20] = 0.0, -1.0                                  # (clusters of one to eight blocks, by the rows' number and length)
    l[6, 1] = np.nan
    l[7] = -np.inf
    if K:
        ids[8] = -1
        ids[10, :] = ids[10, 0]
    rows = [0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 20, 36, 37, 73, 74, N // 2, N - 2, N - 1] if cols < 200000 else [0, 3, 4, 5, 6, 7, 8, 9, N - 1]
    check(l, n, ids, t, 1.3, w, ld=cols + (cols % 3), in_place=True, rows=[r for r in rows if r < N])


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,cols,K", [(74, 65537, 5), (300, 70003, 127), (155, 80001, 0), (90, 66001, 256), (223, 32768, 9), (223, 32767, 257)])
def test_distill_of_many_rows_around_the_forms_limits(dt, N, cols, K):
    test_distill_of_many_rows(dt, N, cols, K)


@pytest.mark.parametrize("cols", [12000, 12160, 12200, 12240, 12280, 12320])
@pytest.mark.parametrize("K", [0, 3])
def test_distill_of_rows_around_48_kb_of_shared_memory(K, cols):
    rng = np.random.default_rng(cols + K)
    l, n, ids, t = batch(rng, 100, cols, max(K, 1), torch.float32)
    check(l, n, ids if K else None, t if K else None, 1.0, None, rows=[0, 1, 50, 99])


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K,few", [(2, 1), (33, 5), (64, 64), (129, 1), (512, 300), (512, 3), (513, 300), (1024, 500), (1024, 2)])
@pytest.mark.parametrize("N,cols", [(3, 2000), (76, 70003)])
def test_distill_of_repeated_entries(dt, N, cols, K, few):
    # few columns for many entries, spread over the row or side by side; left-out ones among them
    rng = np.random.default_rng(1000 * K + few)
    l = (torch.from_numpy(rng.standard_normal((N, cols)).astype(np.float32)) * 2).to(dt)
    ids = np.stack([rng.choice(cols, few, replace=False)[rng.integers(0, few, K)] for _ in range(N)])
    ids[1] = cols - 1 - rng.integers(0, min(few, cols), K)
    ids[2, ::3] = -1
    t = (rng.standard_normal((N, K)) * 2).astype(np.float32)
    t[0, ::5] = -np.inf
    check(l, [cols, cols, cols - 1] + [cols] * (N - 3), ids, t, 1.0, None, rows=[0, 1, 2] + ([40, N - 1] if N > 3 else []))


def test_distill_without_a_teacher_list():
    l = torch.randn(4, 300)
    check(l, [300, 5, 0, 299], None, None, 1.0, None)


def test_distill_of_the_largest_offsets():
    # rows whose offset passes 2^31 elements: strides as a view of a wide buffer has
    N, cols, ld = 5, 1000, (1 << 29) + 17
    buf = torch.empty((N - 1) * ld + cols, dtype=torch.bfloat16, device=DEV)
    l = buf.as_strided((N, cols), (ld, 1))
    rng = np.random.default_rng(1)
    host, n, ids, t = batch(rng, N, cols, 7, torch.bfloat16)
    l.copy_(host)
    args = (torch.tensor(n, dtype=torch.int32, device=DEV), torch.from_numpy(ids.astype(np.int32)).to(DEV), torch.from_numpy(t).to(DEV), 1.0)
    loss, lse = torch.empty(2, N, device=DEV).unbind(0)
    zb.z2z_distill_loss(l, *args, None, loss, lse, l)        # in place
    L, got = f64(host), f64(l)
    for r in range(N):
        row = L[r, :n[r]]
        want_loss, want_lse, want = odis.row(row, ids[r], t[r], 1.0)
        b_loss, b_lse, b_g = bounds(row, ids[r], t[r].astype(np.float64), 1.0, 1.0, torch.bfloat16, want)
        assert abs(loss[r].item() - want_loss) <= b_loss and abs(lse[r].item() - want_lse) <= b_lse
        assert (np.abs(got[r, :n[r]] - want) <= b_g).all() and not got[r, n[r]:].any()


def test_distill_gradient_by_differences():
    rng = np.random.default_rng(4)
    l, n, ids, t = batch(rng, 1, 40, 6, torch.float32, spread=1.0)
    args = (None, torch.from_numpy(ids.astype(np.int32)).to(DEV), torch.from_numpy(t).to(DEV), 2.0)
    g, loss, lse = torch.empty(1, 40, device=DEV), torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    zb.z2z_distill_loss(l.to(DEV), *args, None, loss, lse, g)
    h = 2.0 ** -5
    rows = l.repeat(80, 1)
    for c in range(40):
        rows[2 * c, c] += h
        rows[2 * c + 1, c] -= h
    many = (None, args[1].repeat(80, 1), args[2].repeat(80, 1), 2.0)
    L, e = torch.empty(80, device=DEV), torch.empty(80, device=DEV)
    zb.z2z_distill_loss(rows.to(DEV), *many, None, L, e)
    diff = (L[0::2] - L[1::2]) / (2 * h)
    # the third derivative of T^2 log sum exp(l / T) is at most 1 / T: h^2 / 6 / T; and the loss's own rounding over h
    b = h * h / 6 / 2 + 64 * u * max(1.0, L.abs().max().item()) / h
    assert (diff - g[0]).abs().max().item() <= b


def test_distill_on_two_streams_at_once():
    rng = np.random.default_rng(12)
    jobs = []
    for N, cols, K in ((300, 33003, 16), (200, 50001, 40), (5, 130001, 8)):
        l, n, ids, t = batch(rng, N, cols, K, torch.bfloat16, spread=1.0)
        gl = l.to(DEV)
        args = (gl, torch.tensor(n, dtype=torch.int32, device=DEV), torch.from_numpy(ids.astype(np.int32)).to(DEV), torch.from_numpy(t).to(DEV), 1.0)
        jobs.append((args, N, gl))

    def run(args, N, gl):
        loss, lse = torch.empty(2, N, device=DEV).unbind(0)
        g1, g2 = torch.empty_like(gl), torch.empty_like(gl)
        zb.z2z_distill_loss(*args, None, loss, lse, g1)
        zb.z2z_distill_grad(*args, lse, torch.ones(N, device=DEV), g2)
        return loss, lse, g1, g2

    want = [run(*j) for j in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, j in zip(streams, jobs):
            with torch.cuda.stream(s):
                got.append(run(*j))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_distill_replayed_from_a_graph_on_another_stream():
    rng = np.random.default_rng(6)
    N, cols, K = 9, 20011, 33
    l, n, ids, t = batch(rng, N, cols, K, torch.bfloat16)
    gl, gi, gt = l.to(DEV), torch.from_numpy(ids.astype(np.int32)).to(DEV), torch.from_numpy(t).to(DEV)
    gn = torch.tensor(n, dtype=torch.int32, device=DEV)
    loss, lse = torch.empty(2, N, device=DEV).unbind(0)
    g1, g2 = torch.empty_like(gl), torch.empty_like(gl)
    one = torch.ones(N, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        zb.z2z_distill_loss(gl, gn, gi, gt, 1.0, None, loss, lse, g1)
        zb.z2z_distill_grad(gl, gn, gi, gt, 1.0, lse, one, g2)
    for k in range(3):
        gl.copy_((torch.randn(N, cols) * (k + 1)).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        got = (loss.clone(), lse.clone(), g1.clone(), g2.clone())
        zb.z2z_distill_loss(gl, gn, gi, gt, 1.0, None, loss, lse, g1)
        zb.z2z_distill_grad(gl, gn, gi, gt, 1.0, lse, one, g2)
        assert all(torch.equal(a, b) for a, b in zip(got, (loss, lse, g1, g2)))
        L = f64(gl)
        for r in range(N):
            assert abs(got[0][r].item() - odis.row(L[r, :n[r]], ids[r], t[r], 1.0)[0]) < 1e-3
