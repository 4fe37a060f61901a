"""The operators as a program uses them: a training step from the lookup to the tables' gradients, and beam decoding
with codebooks, caches and the caller's own rows following their beams."""
import copy

import numpy as np
import pytest
import torch

from oracle import beam as obeam, lzw as olzw
from paper_2506_01084_b200 import binding as zb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
u = 2.0 ** -24


def f64(t):
    return t.detach().cpu().double()


@pytest.mark.parametrize("autograd", [False, True])
def test_training_step(autograd):
    """x = s * embed(codes), h = x A, l = h [W_U; U_h], distillation, and back.  Against automatic differentiation in
    fp64; the bound follows the errors of the fp32 steps through the same products on magnitudes."""
    torch.manual_seed(3)
    V, d, cap, B, T, K, scale, temp = 300, 64, 20, 3, 60, 9, 8.0, 1.5
    cb = zb.Codebook(zb.make_config(V, d, 3, cap, B, "fp32", 0, 1, 8), DEV)
    tokens = torch.randint(0, 12, (B, T), dtype=torch.int32, device=DEV)
    codes, after = torch.zeros(2, B, T, dtype=torch.int32, device=DEV).unbind(0)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    zb.z2z_lzw_encode(cb, tokens, torch.tensor([60, 41, 0], dtype=torch.int32, device=DEV), codes, lens, after)
    n_b = zb.z2z_status(cb)[1]
    rows = [(b, i) for b in range(B) for i in range(int(lens[b]))]
    N = len(rows)
    z = torch.stack([codes[b, i] for b, i in rows]).contiguous()
    seq = torch.tensor([b for b, _ in rows], dtype=torch.int32, device=DEV)
    # (a code may be used one position after its entry was made: what row i sees is there once code i is emitted)
    vis = torch.stack([after[b, i] for b, i in rows]).contiguous()
    assert N > 30 and (z >= V).sum() > 5
    WE, WU = torch.randn(V, d, device=DEV) * 0.1, torch.randn(V, d, device=DEV) * 0.3
    Eh, Uh = torch.randn(B, cap, d, device=DEV) * 0.1, torch.randn(B, cap, d, device=DEV) * 0.3
    A = torch.randn(d, d, device=DEV) / 8
    ids = torch.stack([torch.randperm(V + int(k), device=DEV)[:K] for k in vis]).int().contiguous()
    ids[::5, 3:] = -1
    t = torch.randn(N, K, device=DEV) * 2
    w = torch.full((N,), 1.0 / N, device=DEV)
    w[4] = 0.0

    x = torch.empty(N, d, device=DEV)
    zb.z2z_embed_lookup_scaled(cb, z, seq, WE, Eh, scale, x)
    h = x @ A
    logits = torch.full((N, V + cap), float("nan"), device=DEV)
    zb.z2z_dynamic_logits(cb, h, seq, vis, WU, Uh, zb.SELECT_ARGMAX, 1.0, 0, 0, None, None, None, None, logits_debug=logits)
    cols = (V + vis).int()
    loss, lse = torch.empty(2, N, device=DEV).unbind(0)
    if autograd:
        grad = torch.empty_like(logits)
        zb.z2z_distill_loss(logits, cols, ids, t, temp, None, loss, lse)
        zb.z2z_distill_grad(logits, cols, ids, t, temp, lse, w, grad)
    else:
        grad = logits                                        # the logits are not needed any more
        zb.z2z_distill_loss(logits, cols, ids, t, temp, w, loss, lse, grad)
    gh = grad[:, :V] @ WU + torch.einsum("nc,ncd->nd", grad[:, V:], Uh[seq.long()])
    gx = gh @ A.T
    gW, gE = torch.zeros_like(WE), torch.zeros_like(Eh)
    scratch = torch.empty(zb.z2z_embed_grad_scratch_bytes(cb.cfg, N), dtype=torch.uint8, device=DEV)
    zb.z2z_embed_grad(cb, z, seq, gx, scale, True, gW, gE, scratch)
    assert zb.z2z_status(cb)[0].tolist() == [zb.ST_CAP_FROZEN if k == cap else 0 for k in n_b.tolist()]

    W, E, a, wu, uh = (f64(v).requires_grad_(i < 2) for i, v in enumerate((WE, Eh, A, WU, Uh)))
    zc, sc, vc = z.cpu().long(), seq.cpu().long(), vis.cpu().long()
    rows64 = torch.stack([W[c] if c < V else E[b, c - V] for c, b in zip(zc.tolist(), sc.tolist())])
    h64 = scale * rows64 @ a
    total, loss64, q, l64 = 0.0, [], [], []
    for r in range(N):
        M = torch.cat([wu, uh[sc[r], :vc[r]]])
        l = M @ h64[r]
        keep = ids[r].cpu() >= 0
        lp = torch.log_softmax(f64(t[r])[keep] / temp, 0)
        lq = torch.log_softmax(l / temp, 0)
        L = temp ** 2 * (lp.exp() * (lp - lq[ids[r].cpu().long()[keep]])).sum()
        total = total + L * f64(w)[r]
        loss64.append(L.item()); q.append(lq.exp().detach()); l64.append(l.detach())
    total.backward()

    # bounds
    X, Aa = (scale * rows64).abs().detach(), a.abs()
    H = X @ Aa                                               # magnitudes of h
    b_h = (d + 2) * u * H
    gW_b, gE_b = torch.zeros_like(W), torch.zeros_like(E)
    for r in range(N):
        M = torch.cat([wu, uh[sc[r], :vc[r]]]).abs()
        b_l = M @ b_h[r] + (d + 2) * u * (M @ H[r])
        delta = b_l.max().item() / temp
        k = f64(w)[r].item() * temp
        C = M.shape[0]
        p = torch.zeros(C, dtype=torch.float64)
        keep = ids[r].cpu() >= 0
        p.index_add_(0, ids[r].cpu().long()[keep], torch.softmax(f64(t[r])[keep] / temp, 0))
        rel = 2 * delta + (12 * l64[r].abs().max().item() / temp + 200) * u        # (exponentials, normaliser, products)
        b_g = k * (q[r] * rel + p * 200 * u)
        g = k * (q[r] + p)
        assert abs(loss[r].item() - loss64[r]) <= temp ** 2 * (2 * delta + 300 * u * (1 + abs(loss64[r])) + 12 * u * l64[r].abs().max().item())
        b_gh = b_g @ M + (C + 4) * u * (g @ M)
        b_gx = b_gh @ Aa.T + (d + 2) * u * ((g @ M) @ Aa.T)
        gx_m = (g @ M) @ Aa.T
        c, b = int(zc[r]), int(sc[r])
        to = gW_b[c] if c < V else gE_b[b, c - V]
        to += scale * (b_gx + (N + 4) * u * gx_m)
    assert ((f64(gW) - W.grad).abs() <= gW_b).all() and ((f64(gE) - E.grad).abs() <= gE_b).all()
    # (a worst case over some 20 rows of a frequent token and three products: the bound is below a hundredth of the gradient)
    assert W.grad.abs().max() > 100 * gW_b.max()
    # and a step against the gradient changes the loss by its square, to first order (differences of the whole chain)
    eps = 1e-4
    with torch.no_grad():
        def whole(Wv, Ev):
            tot = 0.0
            for r in range(N):
                c, b = int(zc[r]), int(sc[r])
                l = torch.cat([wu, uh[b, :vc[r]]]) @ (scale * (Wv[c] if c < V else Ev[b, c - V]) @ a)
                keep = ids[r].cpu() >= 0
                lp = torch.log_softmax(f64(t[r])[keep] / temp, 0)
                tot += f64(w)[r] * temp ** 2 * (lp.exp() * (lp - torch.log_softmax(l / temp, 0)[ids[r].cpu().long()[keep]])).sum()
            return tot.item()
        dW, dE = f64(gW), f64(gE)
        diff = (whole(W + eps * dW, E + eps * dE) - whole(W - eps * dW, E - eps * dE)) / (2 * eps)
        sq = (dW ** 2).sum().item() + (dE ** 2).sum().item()
        assert abs(diff - sq) <= 1e-3 * sq


def test_beam_decoding():
    torch.manual_seed(11)
    V, d, cap, W, G, M, steps, eos = 60, 16, 24, 3, 3, 3, 14, 5
    B = W * G
    cfg = zb.make_config(V, d, M, cap, B, "fp32", 0, 1, 8)
    cb = zb.Codebook(cfg, DEV)
    WE, WU = torch.randn(V, d, device=DEV), torch.randn(V, d, device=DEV)
    enc = zb.encoder_weights([torch.zeros(M, d, device=DEV)])
    Eh, Uh = torch.zeros(2, B, cap, d, device=DEV).unbind(0)
    # every beam of a request starts from the request's prompt
    prompt = torch.randint(0, 8, (G, 20), dtype=torch.int32, device=DEV).repeat_interleave(W, 0).contiguous()
    codes, lens = torch.zeros_like(prompt), torch.zeros(B, dtype=torch.int32, device=DEV)
    zb.z2z_lzw_encode(cb, prompt, None, codes, lens)
    for side, table, cache in ((zb.CACHE_EMBED, WE, Eh), (zb.CACHE_UNEMBED, WU, Uh)):
        zb.z2z_hyper_embed(cb, side, table, enc, None, None, 0, cache)
    books = []
    for b in range(B):
        books.append(olzw.Codebook(V, M, cap))
        books[b].encode(prompt[b].tolist())
    start = copy.deepcopy(books)
    A = torch.randn(d, d, device=DEV) / 4
    scores = torch.tensor([0.0] + [-np.inf] * (W - 1), device=DEV).repeat(G)
    fin, act = torch.zeros(2, B, dtype=torch.uint8, device=DEV).unbind(0)
    parent, code, new = torch.zeros(3, B, dtype=torch.int32, device=DEV).unbind(0)
    hist = torch.full((B, steps), -9, dtype=torch.int32, device=DEV)
    x = torch.randn(B, d, device=DEV)
    logits = torch.zeros(B, V + cap, device=DEV)
    lse = torch.zeros(B, device=DEV)
    ended_early = moved = 0
    for t in range(steps):
        h = torch.tanh(x @ A) * 1.5
        zb.z2z_dynamic_logits(cb, h, None, None, WU, Uh, zb.SELECT_ARGMAX, 1.0, 0, 0, None, lse, None, None, logits_debug=logits)
        old_s, old_f = scores.cpu().numpy(), fin.cpu().numpy()
        zb.z2z_beam_select(cb, W, logits, lse, scores, fin, eos, parent, code, scores, fin, act)
        L = logits.cpu().numpy()
        want = obeam.select(W, [L[b, :V + books[b].n()] for b in range(B)], lse.cpu().numpy(), old_s, old_f, eos)
        assert parent.tolist() == want[0] and code.tolist() == want[1] and fin.tolist() == want[3] and act.tolist() == want[4]
        assert np.array_equal(scores.cpu().numpy(), np.array(want[2]).astype(np.float32))
        zb.z2z_beam_reorder(cb, parent, Eh, Uh, states=(hist, x))
        books = [copy.deepcopy(books[p]) for p in want[0]]
        start = [start[p] for p in want[0]]
        moved += sum(p != b for b, p in enumerate(want[0]))
        hist[:, t] = code
        zb.z2z_lzw_step(cb, code, act, new)
        for b in range(B):
            assert new[b].item() == (books[b].step(want[1][b]) if want[4][b] else -1)
        for side, table, cache in ((zb.CACHE_EMBED, WE, Eh), (zb.CACHE_UNEMBED, WU, Uh)):
            zb.z2z_hyper_embed(cb, side, table, enc, None, None, B, cache)
        zb.z2z_embed_lookup_scaled(cb, code, None, WE, Eh, 0.5, x)
        ended_early += sum(want[3])
    st, n = zb.z2z_status(cb)
    assert moved > 10 and ended_early > 0
    for b in range(B):
        assert (st[b] & ~zb.ST_CAP_FROZEN) == 0 and n[b] == books[b].n()
        cons, ln = zb.z2z_codebook_read(cb, b)
        assert [tuple(cons[k, :ln[k]].tolist()) for k in range(n[b])] == books[b].entries
        # the slot's history is a stream of its own: its prompt's codebook and its codes give its codebook
        again = copy.deepcopy(start[b])
        for c in hist[b].tolist():
            if c >= 0:
                again.step(c)
        assert again.entries == books[b].entries
        for table, cache in ((WE, Eh), (WU, Uh)):            # rows of the averaging encoder: the mean of at most 3 rows
            for k in range(n[b]):
                rows = f64(table)[list(books[b].entries[k])]
                assert (f64(cache[b, k]) - rows.mean(0)).abs().max() <= 4 * u * rows.abs().max() * 3
