"""Operators around the dynamic vocabulary: their cases, plain forms and 64-bit values.

  embed        input embeddings of a mixed base-token / hypertoken stream, times a scale
  embed_grad   gradient of that lookup for the embedding table and for the hyper-embedding cache
  distill      loss of joint logits against a teacher's top logits, its gradient for the logits
  beam_select  the best continuations of groups of beams over their joint vocabularies, dealt to slots
  beam_reorder the caches and per-sequence rows of surviving beams copied into the slots of beams that died

``run`` computes an operator in elementary torch operations, or (``own``) makes the framework's calls.
Hypertoken counts are functions of the case alone, so that ``work`` knows them; everything else is drawn
from the seed on the GPU.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
NONE = -1                       # a row without a token
EOS = 2                         # base token that ends a beam


def listed():
    return [
        # the input embeddings of one decode step of a small batch: a few rows, latency
        dict(op="embed", name="embed_step_b8", V=128256, d=4096, dtype="bf16", B=8, cap=1024, n=700, N=8, scale=64.0, pad=0.0),
        # the compressed prompts of the default benchmark workload, every code of every sequence
        dict(op="embed", name="embed_prompts", V=128256, d=4096, dtype="bf16", B=32, cap=1024, n=561, N=52800, scale=64.0, pad=0.02),
        # a micro batch of one short text with gradients that add up in fp32 over micro batches
        dict(op="embed_grad", name="embed_grad_micro", V=32064, d=1024, dtype="bf16", grads="fp32", accumulate=True, B=1, cap=1024,
             n=150, N=333, scale=32.0, pad=0.0),
        # a training batch whose tables' gradients are written anew in the tables' type
        dict(op="embed_grad", name="embed_grad_batch", V=128256, d=4096, dtype="bf16", grads="bf16", accumulate=False, B=32, cap=1024,
             n=561, N=52800, scale=64.0, pad=0.02),
        # an fp32 model of an odd width, ragged sequences with padding, gradients that add up
        dict(op="embed_grad", name="embed_grad_fp32_odd", V=50021, d=1000, dtype="fp32", grads="fp32", accumulate=True, B=13, cap=777,
             n=500, N=20011, scale=31.625, pad=0.1),
        # validation loss of a handful of positions on the joint logits as the logits call stores them
        dict(op="distill", name="distill_eval", V=32064, cap=2048, n=682, dtype="fp32", N=32, K=50, temperature=2.0, mode="loss"),
        # a training step of a large vocabulary: loss and gradient in one call, bf16 logits
        dict(op="distill", name="distill_step_bf16", V=128256, cap=4096, n=561, dtype="bf16", N=2048, K=64, temperature=1.0, mode="step"),
        # the two halves as an automatic differentiation calls them, odd row lengths, fp32
        dict(op="distill", name="distill_autograd_fp32", V=128251, cap=4096, n=1416, dtype="fp32", N=700, K=128, temperature=3.0,
             mode="autograd"),
        # one user's beam search of four beams
        dict(op="beam_select", name="beam_select_user", V=32064, cap=2048, n=682, groups=1, beams=4),
        # a serving batch: 32 requests of eight beams
        dict(op="beam_select", name="beam_select_batch", V=128256, cap=4096, n=561, groups=32, beams=8),
        # the caches of one user's four beams after a step in which two of them died
        dict(op="beam_reorder", name="beam_reorder_user", V=32064, d=2048, dtype="bf16", cap=1024, n=300, groups=1, beams=4, M=3, row=256),
        # 12 requests of eight beams with long codebooks
        dict(op="beam_reorder", name="beam_reorder_batch", V=128256, d=4096, dtype="bf16", cap=1024, n=600, groups=12, beams=8, M=4, row=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: widths in steps of 8, any vocabulary, odd lengths, counts over their logarithm."""
    op = rng.choice(["embed", "embed_grad", "embed_grad", "distill", "distill", "beam_select", "beam_select", "beam_reorder"])
    V = _log_int(rng, 500, 128256)
    cap = _log_int(rng, 16, 2048)
    n = rng.randint(0, cap)
    c = dict(op=op, V=V, cap=cap, n=n)
    if op in ("embed", "embed_grad"):
        B = _log_int(rng, 1, 32)
        d = 8 * _log_int(rng, 8, 512)
        c.update(d=d, dtype=rng.choice(["bf16", "bf16", "fp32"]), B=B, scale=round(math.sqrt(d), 3),
                 N=_log_int(rng, max(B, 4), 20000) if op == "embed_grad" else rng.choice([B, _log_int(rng, B, 20000)]),
                 pad=rng.choice([0.0, 0.05, 0.3]))
        if op == "embed_grad":
            c.update(grads=rng.choice(["fp32", c["dtype"]]), accumulate=rng.random() < 0.5, cap=min(cap, 512), n=min(n, 512))
            c["V"] = min(V, 800_000_000 // (d * _size(c["grads"])))
    elif op == "distill":
        N = _log_int(rng, 1, 2048)
        c.update(dtype=rng.choice(["bf16", "fp32"]), N=N, K=_log_int(rng, 1, 256), temperature=rng.choice([0.5, 1.0, 2.0, 4.0]),
                 mode=rng.choice(["loss", "step", "step", "autograd"]), V=min(V, 130_000_000 // N))
    elif op == "beam_select":
        beams = rng.choice([1, 2, 3, 4, 5, 8, 16, 32])
        c.update(beams=beams, groups=_log_int(rng, 1, 256 // beams))
    else:
        beams = rng.choice([2, 3, 4, 5, 8])
        groups = _log_int(rng, 1, 40 // beams)
        c.update(beams=beams, groups=groups, d=8 * _log_int(rng, 8, 512), dtype=rng.choice(["bf16", "fp32"]), cap=min(cap, 1024),
                 n=min(n, 1024), M=rng.randint(2, 5), row=rng.choice([0, 4 * _log_int(rng, 1, 2048)]))
        c["n"] = min(c["n"], c["cap"])
    return c


# ---- what a case fixes ---------------------------------------------------------------------------
def _counts(case, B):
    """Hypertokens of every sequence, ragged around the case's n."""
    return [min(case["cap"], int(case["n"] * (0.6 + 0.8 * ((b * 0.6180339887) % 1.0)))) for b in range(B)]


def _torch_dtype(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def _size(name):
    return 4 if name == "fp32" else 2


def _parents(case):
    """Surviving beams of every group: the first half, at least one; who died takes a survivor's state in turn."""
    W = case["beams"]
    keep = max(1, W // 2)
    return W, keep


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std, dt):
    out = torch.empty(shape, dtype=dt, device=DEV)
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        k = min(1 << 27, flat.numel() - i)
        flat[i:i + k] = torch.randn(k, generator=g, device=DEV) * std
    return out


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _codes(case, g, counts):
    """A mixed stream, sequence after sequence: hypertokens for half of the rows (uniform), base tokens by
    Zipf's law, rows without a token at the end of every sequence's share."""
    N, B, V = case["N"], case["B"], case["V"]
    seq = torch.arange(N, device=DEV) * B // N
    n = torch.tensor(counts, device=DEV)[seq]
    u = torch.rand(3, N, generator=g, device=DEV, dtype=torch.float64)
    rank = torch.exp(u[0] * math.log(V)).long().clamp(1, V) - 1
    base = (rank * 7919 + 13) % V
    hyper = V + (u[1] * n).long()
    z = torch.where((u[2] < 0.5) & (n > 0), hyper, base)
    first = torch.searchsorted(seq, torch.arange(B + 1, device=DEV))
    at = (torch.arange(N, device=DEV) - first[seq]).double() / (first[seq + 1] - first[seq])
    z = torch.where(at >= 1.0 - case["pad"], torch.full_like(z, NONE), z)
    return z.int(), seq.int()


def _session(case, B, counts):
    """The session that a user's program has: its codebooks hold `counts` entries after compressing prompts
    of distinct tokens (every pair is a new entry)."""
    from paper_2506_01084_b200 import binding as zb
    cfg = zb.make_config(case["V"], case.get("d", 8), case.get("M", 3), case["cap"], B, case.get("dtype", "fp32"), 0, 1, 8)
    cb = zb.Codebook(cfg, DEV)
    lens = [c + 1 if c > 0 else 0 for c in counts]
    if max(lens) > 0:
        tokens = ((torch.arange(max(lens), device=DEV)[None, :] + 17 * torch.arange(B, device=DEV)[:, None]) % case["V"]).int()
        codes = torch.empty_like(tokens)
        zb.z2z_lzw_encode(cb, tokens.contiguous(), _i32(lens), codes, torch.empty(B, dtype=torch.int32, device=DEV))
    return cb


def _fit(case):
    """Counts must be below the vocabulary for prompts of distinct tokens."""
    return dict(case, n=min(case["n"], case["V"] // 2))


# ---- inputs ----------------------------------------------------------------------------------------
def _inputs(case, seed):
    case = _fit(case)
    g = _gen(seed)
    s = {"case": case}
    op = case["op"]
    if op in ("embed", "embed_grad"):
        counts = _counts(case, case["B"])
        dt = _torch_dtype(case["dtype"])
        s["counts"] = counts
        s["n"] = _i32(counts)
        s["codes"], s["seq"] = _codes(case, g, counts)
        if op == "embed":
            s["WE"] = _normal(g, (case["V"], case["d"]), 0.02, dt)
            s["Eh"] = _normal(g, (case["B"], case["cap"], case["d"]), 0.05, dt)
        else:
            gt = _torch_dtype(case["grads"])
            s["g"] = _normal(g, (case["N"], case["d"]), 1e-2, dt)
            std = 1.0 if case["accumulate"] else 0.0
            s["gWE"] = _normal(g, (case["V"], case["d"]), std, gt)
            s["gEh"] = _normal(g, (case["B"], case["cap"], case["d"]), std, gt)
    elif op == "distill":
        N, K, cols = case["N"], case["K"], case["V"] + case["cap"]
        counts = _counts(case, 16)
        n_cols = torch.tensor([case["V"] + c for c in counts], device=DEV)[torch.arange(N, device=DEV) * 16 // N]
        # a teacher's columns are distinct: one of each of K equal parts of the row
        part = (n_cols[:, None] // K).clamp(min=1)
        ids = torch.arange(K, device=DEV)[None, :] * part + (torch.rand(N, K, generator=g, device=DEV) * part).long().clamp(max=part - 1)
        t = torch.randn(N, K, generator=g, device=DEV) * 2.0 + 8.0
        # (shorter lists: where the row has fewer columns than K, and a few entries of some rows; row 1 of 2: none)
        gone = (ids >= n_cols[:, None]) | (torch.rand(N, K, generator=g, device=DEV) < 0.05)
        if N > 2:
            gone[1] = True
        logits = _normal(g, (N, cols), 2.0, torch.float32)
        logits.scatter_add_(1, ids.clamp(max=cols - 1), (t + torch.randn(N, K, generator=g, device=DEV)) * 0.8)
        s["logits"] = logits.to(_torch_dtype(case["dtype"]))
        s["n_cols"] = n_cols.int()
        s["ids"] = torch.where(gone, torch.full_like(ids, NONE), ids).int().contiguous()
        s["t"] = t.contiguous()
        # weights of the rows: the mean over the batch; every tenth position is padding
        s["w"] = torch.where(torch.rand(N, generator=g, device=DEV) < 0.1, 0.0, 1.0 / N).float()
    elif op == "beam_select":
        B = case["groups"] * case["beams"]
        counts = _counts(case, B)
        cols = case["V"] + case["cap"]
        s["counts"] = counts
        logits = _normal(g, (B, cols), 2.0, torch.float32)
        peak = torch.randint(0, case["V"], (B, 8), generator=g, device=DEV)
        logits.scatter_add_(1, peak, torch.rand(B, 8, generator=g, device=DEV) * 8.0 + 4.0)
        seen = torch.arange(cols, device=DEV)[None, :] < (case["V"] + torch.tensor(counts, device=DEV))[:, None]
        s["seen"] = seen
        s["logits"] = torch.where(seen, logits, torch.full_like(logits, 100.0))         # (beyond a row's columns: not its logits)
        s["lse"] = torch.logsumexp(torch.where(seen, logits, torch.full_like(logits, -math.inf)).double(), 1).float()
        s["score"] = -20.0 + torch.randn(B, generator=g, device=DEV)
        if case["groups"] > 1:
            s["score"][1:case["beams"]] = -math.inf                                     # a request's first step: one beam is alive
        s["done"] = (torch.rand(B, generator=g, device=DEV) < 0.1).to(torch.uint8)
    else:
        B = case["groups"] * case["beams"]
        counts = _counts(case, B)
        W, keep = _parents(case)
        dt = _torch_dtype(case["dtype"])
        s["counts"] = counts
        s["n"] = _i32(counts)
        s["Eh"] = _normal(g, (B, case["cap"], case["d"]), 0.05, dt)
        s["Uh"] = _normal(g, (B, case["cap"], case["d"]), 0.05, dt)
        s["row"] = torch.randint(0, case["V"], (B, case["row"]), generator=g, device=DEV).int() if case["row"] else None
        # the slots of a group in an order of the seed: the first `keep` stay
        r = random.Random(int(seed))
        parent = list(range(B))
        for q in range(case["groups"]):
            slots = r.sample(range(q * W, (q + 1) * W), W)
            for i, b in enumerate(slots[keep:]):
                parent[b] = slots[i % keep]
        s["parent"] = _i32(parent)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2506_01084_b200 import binding as zb
    case = s["case"]
    op = case["op"]
    if op in ("embed", "embed_grad"):
        s["cb"] = _session(case, case["B"], s["counts"])
        if case["N"] == case["B"]:
            s["seq"] = None                                     # row r belongs to sequence r
        if op == "embed":
            s["out"] = torch.empty(case["N"], case["d"], dtype=s["WE"].dtype, device=DEV)
        else:
            s["scratch"] = torch.empty(zb.z2z_embed_grad_scratch_bytes(s["cb"].cfg, case["N"]), dtype=torch.uint8, device=DEV)
    elif op == "distill":
        s["loss"] = torch.empty(case["N"], dtype=torch.float32, device=DEV)
        s["lse"] = torch.empty_like(s["loss"])
        s["grad"] = torch.empty_like(s["logits"]) if case["mode"] != "loss" else None
    elif op == "beam_select":
        B = s["lse"].numel()
        s["cb"] = _session(case, B, s["counts"])
        s["parent"], s["code"] = torch.empty(2, B, dtype=torch.int32, device=DEV).unbind(0)
        s["next_score"] = torch.empty_like(s["score"])
        s["next_done"], s["active"] = torch.empty(2, B, dtype=torch.uint8, device=DEV).unbind(0)
    else:
        s["cb"] = _session(case, s["n"].numel(), s["counts"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    return (_RUN_OWN if own else _RUN_PLAIN)[case["op"]](s, case)


def _own_embed(s, case):
    from paper_2506_01084_b200 import binding as zb
    zb.z2z_embed_lookup_scaled(s["cb"], s["codes"], s["seq"], s["WE"], s["Eh"], case["scale"], s["out"])
    return s["out"]


def _own_embed_grad(s, case):
    from paper_2506_01084_b200 import binding as zb
    zb.z2z_embed_grad(s["cb"], s["codes"], s["seq"], s["g"], case["scale"], case["accumulate"], s["gWE"], s["gEh"], s["scratch"])
    return {"WE": s["gWE"], "Eh": s["gEh"]}


def _own_distill(s, case):
    from paper_2506_01084_b200 import binding as zb
    T, mode = case["temperature"], case["mode"]
    step = mode == "step"
    zb.z2z_distill_loss(s["logits"], s["n_cols"], s["ids"], s["t"], T, s["w"] if step else None, s["loss"], s["lse"], s["grad"] if step else None)
    if mode == "autograd":
        zb.z2z_distill_grad(s["logits"], s["n_cols"], s["ids"], s["t"], T, s["lse"], s["w"], s["grad"])
    out = {"loss": s["loss"], "lse": s["lse"]}
    return out if mode == "loss" else dict(out, grad=s["grad"])


def _own_beam_select(s, case):
    from paper_2506_01084_b200 import binding as zb
    zb.z2z_beam_select(s["cb"], case["beams"], s["logits"], s["lse"], s["score"], s["done"], EOS, s["parent"], s["code"], s["next_score"],
                       s["next_done"], s["active"])
    return {"parent": s["parent"], "code": s["code"], "score": s["next_score"], "done": s["next_done"], "active": s["active"]}


def _own_beam_reorder(s, case):
    from paper_2506_01084_b200 import binding as zb
    zb.z2z_beam_reorder(s["cb"], s["parent"], s["Eh"], s["Uh"], states=() if s["row"] is None else (s["row"],))
    return {"Eh": s["Eh"], "Uh": s["Uh"], "row": s["row"]} if s["row"] is not None else {"Eh": s["Eh"], "Uh": s["Uh"]}


_RUN_OWN = dict(embed=_own_embed, embed_grad=_own_embed_grad, distill=_own_distill, beam_select=_own_beam_select,
                beam_reorder=_own_beam_reorder)


def _plain_embed(s, case):
    V = case["V"]
    z, b = s["codes"].long(), s["seq"].long()
    hyper = (z >= V)[:, None]
    rows = torch.where(hyper, s["Eh"][b, (z - V).clamp(0, max(case["cap"] - 1, 0))], s["WE"][z.clamp(0, V - 1)]).float()
    rows = torch.where((z >= 0)[:, None], rows * case["scale"], torch.zeros_like(rows))
    return rows.to(s["WE"].dtype)


def _plain_embed_grad(s, case):
    """Sums in 64 bits (a frequent token's has thousands of terms), a block of columns at a time."""
    V, cap, B, d = case["V"], case["cap"], case["B"], case["d"]
    z, b = s["codes"].long(), s["seq"].long()
    base, hyper = ((z >= 0) & (z < V)).nonzero()[:, 0], (z >= V).nonzero()[:, 0]
    to_h = b[hyper] * cap + z[hyper] - V
    there = (torch.arange(cap, device=DEV)[None, :] < s["n"][:, None]).reshape(-1, 1)
    gE = s["gEh"].view(B * cap, d)
    for i in range(0, d, 256):
        j = min(d, i + 256)
        for rows, to, out, own_rows in ((base, z[base], s["gWE"], None), (hyper, to_h, gE, there)):
            acc = torch.zeros(out.shape[0], j - i, dtype=torch.float64, device=DEV)
            acc.index_add_(0, to, s["g"][rows, i:j].double())
            acc *= case["scale"]
            if case["accumulate"]:
                acc += out[:, i:j].double()
            if own_rows is not None:
                acc = torch.where(own_rows, acc, out[:, i:j].double())
            out[:, i:j] = acc.to(torch.float32).to(out.dtype) if out.dtype == torch.float32 else acc.to(out.dtype)
    return {"WE": s["gWE"], "Eh": s["gEh"]}


def _plain_distill(s, case):
    T, N, mode = case["temperature"], case["N"], case["mode"]
    loss = torch.empty(N, device=DEV)
    lse = torch.empty(N, device=DEV)
    grad = torch.empty_like(s["logits"]) if mode != "loss" else None
    col = torch.arange(s["logits"].shape[1], device=DEV)[None, :]
    for i in range(0, N, 256):
        j = min(N, i + 256)
        C = s["n_cols"][i:j].long()[:, None]
        seen = col < C
        l = torch.where(seen, s["logits"][i:j].float(), torch.full((), -math.inf, device=DEV))
        m = l.amax(1, keepdim=True)
        e = torch.exp((l - m) / T)
        tot = e.sum(1, keepdim=True)
        ids = s["ids"][i:j].long()
        there = (ids >= 0) & (ids < C)
        at = ids.clamp(min=0)
        t = torch.where(there, s["t"][i:j], torch.full((), -math.inf, device=DEV))
        tm = t.amax(1, keepdim=True)
        some = tm > -math.inf
        x = torch.where(there, (t - torch.where(some, tm, torch.zeros_like(tm))) / T, torch.full((), -math.inf, device=DEV))
        p = torch.exp(x)
        norm = torch.where(some, p.sum(1, keepdim=True), torch.ones_like(tm))
        p = p / norm
        logq = (l.gather(1, at) - m) / T - torch.log(tot)
        terms = torch.where(there, p * (x - torch.log(norm) - logq), torch.zeros_like(p))
        loss[i:j] = T * T * terms.sum(1)
        lse[i:j] = (m / T + torch.log(tot))[:, 0]
        if grad is not None:
            q = e / tot
            q.scatter_add_(1, at, torch.where(there, -p, torch.zeros_like(p)))
            q = q * (s["w"][i:j, None] * T)
            grad[i:j] = torch.where(seen & some, q, torch.zeros_like(q)).to(grad.dtype)
    out = {"loss": loss, "lse": lse}
    return out if mode == "loss" else dict(out, grad=grad)


def _deal(W, parent, code, score, old_done):
    """The winners of every group, best first, dealt to the group's slots: a parent's best continuation stays in
    the parent's slot, the others go to the slots of beams that have none, in order."""
    G = parent.shape[0]
    i = torch.arange(W, device=parent.device)
    same = parent[:, :, None] == parent[:, None, :]                                        # [group, winner, winner]
    stays = ~(same & (i[None, None, :] < i[None, :, None])).any(2) & (code != -2)
    taken = torch.zeros(G, W + 1, dtype=torch.bool, device=parent.device)
    taken.scatter_(1, torch.where(stays, parent, torch.full_like(parent, W)), True)
    free = ~taken[:, :W]
    # the k-th winner that moves takes the k-th free slot
    order = torch.sort((~free).to(torch.int8), dim=1, stable=True)[1]
    k = torch.cumsum((~stays).long(), 1) - 1
    slot = torch.where(stays, parent, order.gather(1, k.clamp(min=0)))
    return slot


def _plain_beam_select(s, case):
    W, G = case["beams"], case["groups"]
    B, cols = s["logits"].shape
    l = torch.where(s["seen"], s["logits"], torch.full((), -math.inf, device=DEV))
    top, col = torch.sort(l, dim=1, descending=True, stable=True)
    w = min(W, cols)
    top, col = top[:, :w], col[:, :w]
    score = s["score"].double()[:, None] + (top.double() - s["lse"].double()[:, None])
    done = s["done"].bool()[:, None]
    first = torch.arange(w, device=DEV)[None, :] == 0
    score = torch.where(done, torch.where(first, s["score"].double()[:, None], torch.full((), -math.inf, device=DEV, dtype=torch.float64)), score)
    col = torch.where(done, torch.full_like(col, NONE), col)
    best, at = torch.sort(score.view(G, W * w), dim=1, descending=True, stable=True)
    best, at = best[:, :W], at[:, :W]
    beam = at // w
    code = col.view(G, W * w).gather(1, at)
    dead = ~(best > -math.inf)
    # slots without a continuation keep what they hold
    code = torch.where(dead, torch.full_like(code, -2), code)
    slot = _deal(W, torch.where(dead, torch.full_like(beam, W), beam), code, best, None)
    here = torch.arange(G, device=DEV)[:, None] * W
    parent = torch.where(dead, here + slot, here + beam).int()
    ended = done.view(G, W).gather(1, torch.where(dead, slot, beam))
    out = {}
    for name, v, dt in (("parent", parent, torch.int32), ("code", torch.where(dead, torch.full_like(code, NONE), code), torch.int32),
                        ("score", best, torch.float32), ("done", dead | ended | (code == EOS), torch.uint8),
                        ("active", ~dead & ~ended, torch.uint8)):
        out[name] = torch.empty(G, W, dtype=dt, device=DEV).scatter_(1, slot, v.to(dt)).view(-1)
    return out


def _plain_beam_reorder(s, case):
    p = s["parent"].long()
    moved = p != torch.arange(p.numel(), device=DEV)
    rows = (torch.arange(case["cap"], device=DEV)[None, :] < s["n"][p][:, None]) & moved[:, None]
    for name in ("Eh", "Uh"):
        s[name].copy_(torch.where(rows[:, :, None], s[name][p], s[name]))
    if s["row"] is None:
        return {"Eh": s["Eh"], "Uh": s["Uh"]}
    s["row"].copy_(s["row"][p])
    return {"Eh": s["Eh"], "Uh": s["Uh"], "row": s["row"]}


_RUN_PLAIN = dict(embed=_plain_embed, embed_grad=_plain_embed_grad, distill=_plain_distill, beam_select=_plain_beam_select,
                  beam_reorder=_plain_beam_reorder)


# ---- what a pass cannot do without -----------------------------------------------------------------------
def _distinct_rows(case, counts):
    """Rows of the two tables that the codes of a case name, as expected from their distribution."""
    N, V, B = case["N"] * (1.0 - case["pad"]), case["V"], case["B"]
    r = np.arange(1, V + 1, dtype=np.float64)
    p = np.log((r + 1) / r) / math.log(V)
    some = np.array(counts) > 0
    base = N * (1.0 - 0.5 * some.mean())
    got = float(np.sum(1.0 - np.exp(base * np.log1p(-np.minimum(p, 0.999)))))
    for c in counts:
        if c > 0:
            got += c * (1.0 - math.exp(-0.5 * N / B / c))
    return got


def work(case):
    case = _fit(case)
    op = case["op"]
    if op == "embed":
        row = case["d"] * _size(case["dtype"])
        counts = _counts(case, case["B"])
        return {"bytes": _distinct_rows(case, counts) * row + case["N"] * (row + 8), "flops": case["N"] * case["d"]}
    if op == "embed_grad":
        counts = _counts(case, case["B"])
        rows = 2 * _distinct_rows(case, counts) if case["accumulate"] else case["V"] + sum(counts)
        return {"bytes": case["N"] * (case["d"] * _size(case["dtype"]) * (1.0 - case["pad"]) + 8) + rows * case["d"] * _size(case["grads"]),
                "flops": case["N"] * case["d"] + rows * case["d"]}
    if op == "distill":
        cols = case["V"] + sum(_counts(case, 16)) / 16
        e = _size(case["dtype"])
        per = cols * e + case["K"] * 8 + 16
        if case["mode"] != "loss":
            per += (case["V"] + case["cap"]) * e
        return {"bytes": case["N"] * per, "flops": case["N"] * cols * (4 if case["mode"] == "loss" else 6)}
    B = case["groups"] * case["beams"]
    counts = _counts(case, B)
    if op == "beam_select":
        return {"bytes": sum(4.0 * (case["V"] + c) + 30 for c in counts), "flops": sum(case["V"] + c for c in counts)}
    W, keep = _parents(case)
    mean = sum(counts) / B
    slots = 64
    while slots < 2 * case["cap"]:
        slots *= 2
    state = 2 * mean * case["d"] * _size(case["dtype"]) + mean * (4 * case["M"] + 1) + 8 * slots + 4 * case["row"]
    return {"bytes": 2.0 * case["groups"] * (W - keep) * state, "flops": 0}


# ---- 64-bit values ---------------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    case = s["case"]
    return _EXACT[case["op"]](s, case)


def _exact_embed(s, case):
    """Row by row from one table of 64-bit rows: those that the codes name, first the tokens', then the entries'."""
    z, b = s["codes"].long(), s["seq"].long()
    out = torch.zeros(case["N"], case["d"], dtype=torch.float64, device=DEV)
    tok, ent = (z >= 0) & (z < case["V"]), z >= case["V"]
    out[tok] = s["WE"].index_select(0, z[tok]).double() * case["scale"]
    if ent.any():
        out[ent] = s["Eh"].view(-1, case["d"]).index_select(0, b[ent] * case["cap"] + z[ent] - case["V"]).double() * case["scale"]
    return out


def _exact_embed_grad(s, case):
    """Differences of running sums over the rows in the order of their targets."""
    V, cap, B, d = case["V"], case["cap"], case["B"], case["d"]
    z, b = s["codes"].cpu().numpy().astype(np.int64), s["seq"].cpu().numpy().astype(np.int64)
    target = np.where(z < V, z, V + b * cap + z - V)
    rows = np.flatnonzero(z >= 0)
    rows = rows[np.argsort(target[rows], kind="stable")]
    names, start = np.unique(target[rows], return_index=True)
    end = torch.from_numpy(np.append(start[1:], rows.size) - 1).to(DEV)
    rows, names = torch.from_numpy(rows).to(DEV), torch.from_numpy(names).to(DEV)
    full = torch.empty(V + B * cap, d, dtype=torch.float64, device=DEV)
    if case["accumulate"]:
        full[:V], full[V:] = s["gWE"], s["gEh"].view(-1, d)
    else:
        full.zero_()
        full[V:] = torch.where((torch.arange(cap, device=DEV)[None, :] < s["n"][:, None]).view(-1, 1), full[V:], s["gEh"].view(-1, d).double())
    for i in range(0, d, 512):
        j = min(d, i + 512)
        run_sum = torch.cumsum(s["g"][:, i:j].index_select(0, rows).double(), 0).index_select(0, end)
        run_sum[1:] -= run_sum[:-1].clone()
        full[:, i:j].index_add_(0, names, run_sum * case["scale"])
    return {"WE": full[:V], "Eh": full[V:].view(B, cap, d)}


def _exact_distill(s, case):
    """Row by row on the row's own columns and the teacher's present entries."""
    T, N, mode = case["temperature"], case["N"], case["mode"]
    if N * s["logits"].shape[1] > 400_000_000:
        return None
    loss, lse = torch.zeros(2, N, dtype=torch.float64, device=DEV).unbind(0)
    grad = torch.zeros(s["logits"].shape, dtype=torch.float64, device=DEV) if mode != "loss" else None
    cols, ids = s["n_cols"].tolist(), s["ids"].cpu()
    for r in range(N):
        C = cols[r]
        lq = torch.log_softmax(s["logits"][r, :C].double() / T, 0)
        lse[r] = torch.logsumexp(s["logits"][r, :C].double() / T, 0)
        k = ((ids[r] >= 0) & (ids[r] < C)).nonzero()[:, 0].to(DEV)
        if not k.numel():
            continue
        at = s["ids"][r].long().index_select(0, k)
        lp = torch.log_softmax(s["t"][r].index_select(0, k).double() / T, 0)
        loss[r] = T * T * (lp.exp() * (lp - lq[at])).sum()
        if grad is not None:
            d = lq.exp()
            d.index_add_(0, at, -lp.exp())
            grad[r, :C] = d * T * s["w"][r].double()
    out = {"loss": loss, "lse": lse}
    return out if mode == "loss" else dict(out, grad=grad)


def _exact_beam_select(s, case):
    """Group by group on the host: every candidate that is at least as good as the W-th."""
    W, G, V = case["beams"], case["groups"], case["V"]
    l = s["logits"].cpu().numpy()
    lse, score = s["lse"].cpu().numpy().astype(np.float64), s["score"].cpu().numpy().astype(np.float64)
    done = s["done"].cpu().numpy()
    B = G * W
    parent, code = np.arange(B, dtype=np.int64), np.full(B, NONE, dtype=np.int64)
    new, ended, active = np.full(B, -np.inf), np.ones(B, dtype=np.int64), np.zeros(B, dtype=np.int64)
    for q in range(G):
        cand = []
        for b in range(q * W, (q + 1) * W):
            if score[b] == -np.inf:
                continue
            if done[b]:
                cand.append((-score[b], b, 0.0, NONE))
                continue
            row = l[b, :V + s["counts"][b]].astype(np.float64)
            k = min(W, row.size)
            for c in np.flatnonzero(row >= -np.partition(-row, k - 1)[k - 1]).tolist():
                cand.append((-(score[b] + (row[c] - lse[b])), b, -row[c], c))
        cand.sort()
        won = cand[:W]
        kept, rest = {}, []
        for w in won:
            if w[1] in kept:
                rest.append(w)
            else:
                kept[w[1]] = w
        free = [b for b in range(q * W, (q + 1) * W) if b not in kept]
        for b, w in list(kept.items()) + list(zip(free, rest)):
            parent[b], code[b], new[b] = w[1], w[3], -w[0]
            ended[b] = 1 if done[w[1]] or w[3] == EOS else 0
            active[b] = 0 if done[w[1]] else 1
    i = lambda v: torch.from_numpy(v).to(DEV)  # noqa: E731
    return {"parent": i(parent), "code": i(code), "score": i(new), "done": i(ended), "active": i(active)}


def _exact_beam_reorder(s, case):
    """Copies: sequence after sequence."""
    out = {k: s[k].double().clone() for k in ("Eh", "Uh")}
    if s["row"] is not None:
        out["row"] = s["row"].clone()
    for b, p in enumerate(s["parent"].tolist()):
        if p != b:
            for k in ("Eh", "Uh"):
                out[k][b, :s["counts"][p]] = s[k][p, :s["counts"][p]].double()
            if s["row"] is not None:
                out["row"][b] = s["row"][p]
    return out


_EXACT = dict(embed=_exact_embed, embed_grad=_exact_embed_grad, distill=_exact_distill, beam_select=_exact_beam_select,
              beam_reorder=_exact_beam_reorder)
