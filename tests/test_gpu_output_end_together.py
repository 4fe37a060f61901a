"""The operators of a training step as a program uses them: next-code prediction on compressed sequences, from the scaled
lookup through the joint cross entropy to the tables' gradients, summed over micro batches, and their clipping."""
import numpy as np
import pytest
import torch

from oracle import xent as ox
from paper_2506_01084_b200 import binding as zb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24


def f64(t):
    return t.detach().cpu().double()


@pytest.mark.parametrize("in_place", [False, True])
def test_training_step(in_place):
    """x = s E[codes], l = x [W_U; U_h], cross entropy against the next code over the entries that exist by then."""
    torch.manual_seed(11)
    V, d, cap, B, T, s = 150, 32, 24, 4, 80, 4.0
    cb = zb.Codebook(zb.make_config(V, d, 3, cap, B, "fp32", 0, 1, 8), DEV)
    tokens = torch.randint(0, 9, (B, T), dtype=torch.int32, device=DEV)
    codes, after = torch.zeros(2, B, T, dtype=torch.int32, device=DEV).unbind(0)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    zb.z2z_lzw_encode(cb, tokens, torch.tensor([80, 51, 0, 2], dtype=torch.int32, device=DEV), codes, lens, after)
    n_b = zb.z2z_status(cb)[1]
    rows = [(b, i) for b in range(B) for i in range(int(lens[b]))]
    batches = [rows[0::2], rows[1::2]]
    WE, WU = torch.randn(V, d, device=DEV) * 0.2, torch.randn(V, d, device=DEV) * 0.4
    Eh, Uh = torch.randn(B, cap, d, device=DEV) * 0.2, torch.randn(B, cap, d, device=DEV) * 0.4
    grads = {k: torch.zeros_like(t) for k, t in (("WE", WE), ("Eh", Eh), ("WU", WU), ("Uh", Uh))}

    W64, E64, wu64, uh64 = (f64(t).requires_grad_() for t in (WE, Eh, WU, Uh))
    total = 0.0
    tol = {k: np.zeros(t.shape) for k, t in grads.items()}
    for batch in batches:
        N = len(batch)
        assert N > 20
        pick = lambda t, at: torch.stack([t[b, i] for b, i in at]).contiguous()  # noqa: E731
        z, vis = pick(codes, batch), pick(after, batch)
        seq = torch.tensor([b for b, _ in batch], dtype=torch.int32, device=DEV)
        target = torch.tensor([int(codes[b, i + 1]) if i + 1 < int(lens[b]) else -1 for b, i in batch], dtype=torch.int32, device=DEV)
        assert int((target >= V).sum()) > 3 and int((target < 0).sum()) > 0
        x = torch.empty(N, d, device=DEV)
        zb.z2z_embed_lookup_scaled(cb, z, seq, WE, Eh, s, x)
        loss, lse = torch.empty(2, N, device=DEV).unbind(0)
        w = torch.full((N,), 1.0 / N, device=DEV)
        gx = torch.empty_like(x)
        scratch = torch.empty(zb.z2z_xent_scratch_bytes(cb.cfg, N, torch.float32)[1], dtype=torch.uint8, device=DEV)
        zb.z2z_xent_step(cb, x, seq, vis, WU, Uh, target, w, loss, lse, True, gx, grads["WU"], grads["Uh"], scratch)
        scratch = torch.empty(zb.z2z_embed_grad_scratch_bytes(cb.cfg, N), dtype=torch.uint8, device=DEV)
        zb.z2z_embed_grad(cb, z, seq, gx, s, True, grads["WE"], grads["Eh"], scratch)

        zc, sc, vc, tc = (t.cpu().long() for t in (z, seq, vis, target))
        x64 = s * torch.stack([W64[c] if c < V else E64[b, c - V] for c, b in zip(zc.tolist(), sc.tolist())])
        for r in range(N):
            if tc[r] >= 0:
                l = torch.cat([wu64, uh64[sc[r], :vc[r]]]) @ x64[r]
                total = total + torch.nn.functional.cross_entropy(l[None], tc[r][None]) / N
        # bounds: what the cross entropy's own test allows for the rows as they are, through the sums that follow
        o = ox.cross_entropy(x.cpu().double().numpy(), sc.numpy(), vc.numpy(), f64(WU).numpy(), f64(Uh).numpy(), n_b.tolist(), tc.numpy(), np.full(N, 1 / N))
        e_l = ((d + 8) * 2 * U32 + 8 * U32) * o["size"].max() + 2 * U32 * o["size"].max()       # (and x's own rounding)
        rel = 2.0 ** -23 + 2 * e_l + 2 * U32 * np.abs(o["lse"]).max() + (64 + V / 64) * U32 + 2.0 ** -21 + 2.0 ** -20 + 2 * U32
        for k in ("WU", "Uh"):
            tol[k] += (rel + (N + 16) * 2 * U32) * o["abs_" + k]
        each = (rel + (V + cap + 16) * 2 * U32) * o["abs_hidden"]
        for r in range(N):
            add = s * (each[r] + (N + 2) * U32 * o["abs_hidden"][r])
            if zc[r] < V:
                tol["WE"][zc[r]] += add
            else:
                tol["Eh"][sc[r], zc[r] - V] += add
    total.backward()
    want = {"WE": W64.grad, "Eh": E64.grad, "WU": wu64.grad, "Uh": uh64.grad}
    for k in want:
        tol[k] += 4 * U32 * want[k].abs().numpy() + 1e-30
        off = (f64(grads[k]) - want[k]).abs().numpy()
        assert np.all(off <= tol[k]), (k, off.max(), np.max(off / tol[k]))
    assert not any(v & ~zb.ST_CAP_FROZEN for v in zb.z2z_status(cb)[0].tolist())

    # the mean over the micro batches, clipped to a fifth of its norm; hypertokens' gradients belong to no parameter
    names = ["WE", "WU"]
    norm64 = 0.5 * float(torch.sqrt(sum((want[k] ** 2).sum() for k in names)))
    e_norm = 0.5 * float(np.sqrt(sum((tol[k] ** 2).sum() for k in names))) + 6 * U32 * norm64
    outs = [grads[k] if in_place else torch.empty(grads[k].shape, dtype=torch.bfloat16, device=DEV) for k in names]
    lst = zb.grad_tensors([grads[k] for k in names], outs)
    norm = torch.empty(1, device=DEV)
    scratch = torch.empty(zb.z2z_grad_clip_scratch_bytes(lst), dtype=torch.uint8, device=DEV)
    most = norm64 / 5
    zb.z2z_grad_clip(lst, 0.5, most, norm, scratch)
    assert abs(norm.item() - norm64) <= e_norm
    factor = 0.5 * most / (norm64 + 1e-6)
    for k, out in zip(names, outs):
        y = factor * want[k].numpy()
        step = U32 if in_place else 2.0 ** -8
        bound = factor * tol[k] * 1.01 + np.abs(y) * (1.01 * e_norm / norm64 + 6 * U32 + step) + 2.0 ** -133
        off = np.abs(f64(out).numpy() - y)
        assert np.all(off <= bound), (k, off.max(), np.max(off / bound))


def test_one_graph_of_the_whole_step():
    """Loss, gradients and clipping captured together and replayed on new inputs."""
    torch.manual_seed(2)
    V, d, cap, B, N = 400, 64, 16, 3, 90
    cb = zb.Codebook(zb.make_config(V, d, 3, cap, B, "bf16", 0, 1, 8), DEV)
    tokens = torch.randint(0, 8, (B, 40), dtype=torch.int32, device=DEV)
    zb.z2z_lzw_encode(cb, tokens, torch.tensor([40, 9, 1], dtype=torch.int32, device=DEV), torch.empty_like(tokens), torch.empty(B, dtype=torch.int32, device=DEV))
    n = zb.z2z_status(cb)[1]
    seq = torch.randint(0, B, (N,), dtype=torch.int32, device=DEV)
    hidden, target = torch.zeros(N, d, dtype=torch.bfloat16, device=DEV), torch.zeros(N, dtype=torch.int32, device=DEV)
    WU, Uh = ((torch.randn(*x, device=DEV) * 0.2).bfloat16() for x in ((V, d), (B, cap, d)))
    loss, lse = torch.empty(2, N, device=DEV).unbind(0)
    gh, gW, gU = torch.empty_like(hidden), torch.empty(V, d, device=DEV), torch.empty(B, cap, d, device=DEV)
    out, norm = torch.empty(V, d, dtype=torch.bfloat16, device=DEV), torch.empty(1, device=DEV)
    lst = zb.grad_tensors([gW], [out])
    s1 = torch.empty(zb.z2z_xent_scratch_bytes(cb.cfg, N, torch.float32)[1], dtype=torch.uint8, device=DEV)
    s2 = torch.empty(zb.z2z_grad_clip_scratch_bytes(lst), dtype=torch.uint8, device=DEV)

    def step():
        zb.z2z_xent_step(cb, hidden, seq, None, WU, Uh, target, None, loss, lse, False, gh, gW, gU, s1)
        zb.z2z_grad_clip(lst, 1.0 / N, 0.05, norm, s2)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        hidden.copy_(torch.randn(N, d, device=DEV))
        target.copy_((torch.rand(N, device=DEV) * (V + n.to(DEV)[seq.long()])).int())
        target[k::5] = -1
        step()
        want = [t.clone() for t in (loss, lse, gh, gW, out, norm)]
        for t in (loss, lse, gh, gW, out, norm):
            t.fill_(5.0)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((loss, lse, gh, gW, out, norm), want))
