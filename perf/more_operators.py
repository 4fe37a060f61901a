"""Operators of a training step at the output end: their cases, plain forms and 64-bit values.

  xent   cross entropy over the joint vocabulary [W_U; U_h of the row's sequence] from hidden rows, without stored logits:
         the losses alone (mode loss), losses and the gradients of hidden rows, W_U and U_h in one call (step), or in the
         two calls that an automatic differentiation makes (autograd)
  clip   the global norm of many gradient tensors, and the tensors scaled to a largest norm

``run`` computes an operator in elementary torch operations, or (``own``) makes the framework's calls.  Hypertoken
counts and which rows count are functions of the case alone, so that ``work`` knows them; everything else is drawn from
the seed on the GPU.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
NONE = -1                       # a row without a target
MAX_NORM = 1.0


def listed():
    return [
        # validation loss of a few dozen positions of one text
        dict(op="xent", name="xent_eval_text", mode="loss", V=32064, d=2048, dtype="bf16", B=1, cap=1024, n=300, N=61, skip=0.0,
             causal=True, order="sequences"),
        # validation loss of a batch of prompts
        dict(op="xent", name="xent_eval_batch", mode="loss", V=128256, d=4096, dtype="bf16", B=16, cap=1024, n=561, N=2047, skip=0.1,
             causal=True, order="sequences"),
        # a micro batch of short texts whose gradients add up in fp32 over micro batches
        dict(op="xent", name="xent_step_micro", mode="step", V=32064, d=1024, dtype="bf16", B=3, cap=1024, n=150, N=333, skip=0.0,
             causal=False, order="sequences", grads="fp32", accumulate=True, weights="mean"),
        # a few answers of a preference or reward step on a large vocabulary: the tables are the work
        dict(op="xent", name="xent_step_few", mode="step", V=128256, d=4096, dtype="bf16", B=4, cap=1024, n=200, N=48, skip=0.0,
             causal=False, order="sequences", grads="bf16", accumulate=False, weights="mean"),
        # a training batch, prompts masked, the tables' gradients written anew in the tables' type
        dict(op="xent", name="xent_step_batch", mode="step", V=128256, d=4096, dtype="bf16", B=16, cap=1024, n=561, N=4096, skip=0.1,
             causal=True, order="sequences", grads="bf16", accumulate=False, weights="mean"),
        # the two halves as an automatic differentiation calls them: odd width, a third of the rows masked, every
        # sequence's mean, rows of all sequences in turn
        dict(op="xent", name="xent_autograd_odd", mode="autograd", V=50021, d=1000, dtype="bf16", B=13, cap=777, n=500, N=1777, skip=0.3,
             causal=True, order="turns", grads="bf16", accumulate=True, weights="sequence"),
        # an fp32 model
        dict(op="xent", name="xent_step_fp32", mode="step", V=8009, d=520, dtype="fp32", B=5, cap=300, n=200, N=1021, skip=0.1,
             causal=True, order="sequences", grads="fp32", accumulate=False, weights="mean"),
        # the gradients of a small fp32 hyper-encoder pair, clipped into buffers of their own: latency
        dict(op="clip", name="clip_tiny", V=512, d=64, dff=256, layers=2, tables=True, dtype="fp32", out="fp32", scale=1.0, norm=4.0, shift=0),
        # fp32 sums over micro batches, divided by their number, clipped and rounded for a bf16 optimiser
        dict(op="clip", name="clip_sums_to_bf16", V=32064, d=2048, dff=8192, layers=2, tables=True, dtype="fp32", out="bf16", scale=0.125,
             norm=3.0, shift=0),
        # all gradients of a large head and its encoders in place, below the largest norm: the norm is the work
        dict(op="clip", name="clip_below_in_place", V=128256, d=4096, dff=16384, layers=2, tables=True, dtype="bf16", out="same", scale=1.0,
             norm=0.5, shift=0),
        # bf16 gradients that are odd pieces of a flat buffer
        dict(op="clip", name="clip_odd_pieces", V=50021, d=1000, dff=4000, layers=3, tables=True, dtype="bf16", out="bf16", scale=1.0, norm=2.5,
             shift=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: widths in steps of 8, any vocabulary, odd lengths, counts over their logarithm."""
    if rng.random() < 0.35:
        d = 8 * _log_int(rng, 4, 256)
        dtype = rng.choice(["bf16", "fp32"])
        return dict(op="clip", V=_log_int(rng, 500, 64000), d=d, dff=4 * d, layers=rng.randint(1, 4), tables=rng.random() < 0.5, dtype=dtype,
                    out=rng.choice(["same", "bf16", "fp32"]), scale=rng.choice([1.0, 1.0, 0.25]), norm=rng.choice([0.5, 3.0, 20.0]),
                    shift=rng.choice([0, 0, 1, 5]))
    mode = rng.choice(["loss", "step", "step", "autograd"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    cap = _log_int(rng, 16, 1024)
    c = dict(op="xent", mode=mode, V=_log_int(rng, 500, 128256), d=8 * _log_int(rng, 8, 512), dtype=dtype, B=_log_int(rng, 1, 32), cap=cap,
             n=rng.randint(0, cap), N=_log_int(rng, 4, 4096), skip=rng.choice([0.0, 0.1, 0.4]), causal=rng.random() < 0.5,
             order=rng.choice(["sequences", "sequences", "turns"]))
    if dtype == "fp32":
        c.update(V=min(c["V"], 16000), d=min(c["d"], 1024), N=min(c["N"], 2048))
    if mode != "loss":
        c.update(grads="fp32" if dtype == "fp32" else rng.choice(["bf16", "bf16", "fp32"]), accumulate=rng.random() < 0.5,
                 weights=rng.choice(["mean", "sequence"]))
    return c


# ---- what a case fixes ---------------------------------------------------------------------------
def _counts(case):
    """Hypertokens of every sequence, ragged around the case's n; their entries come from distinct tokens."""
    n = min(case["n"], case["V"] // 2)
    return [min(case["cap"], int(n * (0.6 + 0.8 * ((b * 0.6180339887) % 1.0)))) for b in range(case["B"])]


def _rows(case):
    """(sequence, hypertokens it sees, whether it counts) of every row; the first rows of a sequence are its prompt
    and have no target."""
    N, B = case["N"], case["B"]
    r = torch.arange(N)
    seq = r * B // N if case["order"] == "sequences" else r % B
    size = torch.bincount(seq, minlength=B)
    first = torch.cumsum(size, 0) - size
    place = r - first[seq] if case["order"] == "sequences" else r // B
    at = (place.double() + 1.0) / size[seq].double()
    n = torch.tensor(_counts(case))[seq]
    sees = (n.double() * at).long() if case["causal"] else n
    return seq, sees, at > case["skip"]


def _torch_dtype(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def _size(name):
    return 4 if name == "fp32" else 2


def _shapes(case):
    """Shapes of the gradients: both tables, and the tensors of two encoders."""
    d, dff = case["d"], case["dff"]
    layer = [(d,), (d,), (3 * d, d), (3 * d,), (d, d), (d,), (d,), (d,), (dff, d), (dff,), (d, dff), (d,)]
    return ([(case["V"], d)] * 2 if case["tables"] else []) + ([(3, d)] + layer * case["layers"]) * 2


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


def _session(case, counts):
    """The session that a user's program has: its codebooks hold `counts` entries after compressing prompts
    of distinct tokens (every pair is a new entry)."""
    from paper_2506_01084_b200 import binding as zb
    B = case["B"]
    cb = zb.Codebook(zb.make_config(case["V"], case["d"], 3, case["cap"], B, case["dtype"], 0, 1, 8), DEV)
    lens = [c + 1 if c > 0 else 0 for c in counts]
    if max(lens) > 0:
        tokens = ((torch.arange(max(lens), device=DEV)[None, :] + 17 * torch.arange(B, device=DEV)[:, None]) % case["V"]).int()
        codes = torch.empty_like(tokens)
        zb.z2z_lzw_encode(cb, tokens.contiguous(), torch.tensor(lens, dtype=torch.int32, device=DEV), codes,
                          torch.empty(B, dtype=torch.int32, device=DEV))
    return cb


# ---- inputs ----------------------------------------------------------------------------------------
def _inputs(case, seed):
    return (_xent_inputs if case["op"] == "xent" else _clip_inputs)(case, _gen(seed))


def _xent_inputs(case, g):
    N, B, V, d, cap = (case[k] for k in ("N", "B", "V", "d", "cap"))
    dt = _torch_dtype(case["dtype"])
    counts = _counts(case)
    seq, sees, counted = (t.to(DEV) for t in _rows(case))
    s = {"case": case, "counts": counts, "seq": seq.int(), "sees": sees.int() if case["causal"] else None, "counted": counted}
    std = 1.3 / math.sqrt(d)
    s["WU"] = _normal(g, (V, d), std, dt)
    s["Uh"] = _normal(g, (B, cap, d), std, dt)
    # targets: hypertokens for a third of the rows that see any, base tokens by Zipf's law
    u = torch.rand(4, N, generator=g, device=DEV, dtype=torch.float64)
    base = ((torch.exp(u[0] * math.log(V)).long().clamp(1, V) - 1) * 7919 + 13) % V
    target = torch.where((u[2] < 0.33) & (sees > 0), V + (u[1] * sees).long(), base)
    s["target"] = torch.where(counted, target, torch.full_like(target, NONE)).int()
    # hidden rows that know their target more or less well: it gets up to 14 nats
    hyper = (target >= V)[:, None]
    row = torch.where(hyper, s["Uh"].view(-1, d)[seq * cap + (target - V).clamp(0, cap - 1)], s["WU"][target.clamp(max=V - 1)]).float()
    s["hidden"] = (_normal(g, (N, d), 1.0, torch.float32) + row * (u[3].float() * 8.0)[:, None]).to(dt)
    if case["mode"] == "loss":
        return s
    per = torch.bincount(seq[counted], minlength=B).clamp(min=1)
    live = int((torch.bincount(seq[counted], minlength=B) > 0).sum())
    s["w"] = (torch.full((N,), 1.0 / max(1, int(counted.sum())), device=DEV) if case["weights"] == "mean"
              else (1.0 / (per[seq].double() * max(1, live))).float())
    gt = _torch_dtype(case["grads"])
    scale = 1e-3 if case["accumulate"] else 0.0
    s["gWU"], s["gUh"] = _normal(g, (V, d), scale, gt), _normal(g, (B, cap, d), scale, gt)
    return s


def _pieces(flat, case):
    """The tensors of a case as pieces of one flat buffer, `shift` elements apart."""
    out, at = [], 0
    for x in _shapes(case):
        at += case["shift"]
        out.append(flat[at:at + math.prod(x)].view(x))
        at += math.prod(x)
    return out


def _clip_inputs(case, g):
    sizes = [math.prod(x) for x in _shapes(case)]
    total = sum(sizes) + case["shift"] * len(sizes)
    flat = _normal(g, (total,), case["norm"] / (case["scale"] * math.sqrt(sum(sizes))), _torch_dtype(case["dtype"]))
    out = flat if case["out"] == "same" else torch.zeros(total, dtype=_torch_dtype(case["out"]), device=DEV)
    return {"case": case, "out": out, "grads": _pieces(flat, case), "outs": _pieces(out, case)}


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2506_01084_b200 import binding as zb
    if case["op"] == "clip":
        s["norm"] = torch.empty(1, dtype=torch.float32, device=DEV)
        s["list"] = zb.grad_tensors(s["grads"], s["outs"])
        s["scratch"] = torch.empty(zb.z2z_grad_clip_scratch_bytes(s["list"]), dtype=torch.uint8, device=DEV)
        return s
    s["cb"] = _session(case, s["counts"])
    s["loss"], s["lse"] = torch.empty(2, case["N"], dtype=torch.float32, device=DEV).unbind(0)
    if case["mode"] != "loss":
        s["gh"] = torch.empty_like(s["hidden"])
    most = zb.z2z_xent_scratch_bytes(s["cb"].cfg, case["N"], None if case["mode"] == "loss" else s["gWU"].dtype)[1]
    s["scratch"] = torch.empty(most, dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if case["op"] == "clip":
        return _own_clip(s, case) if own else _plain_clip(s, case)
    return _own_xent(s, case) if own else _plain_xent(s, case)


def _own_xent(s, case):
    from paper_2506_01084_b200 import binding as zb
    args = (s["cb"], s["hidden"], s["seq"], s["sees"], s["WU"], s["Uh"], s["target"])
    if case["mode"] == "step":
        zb.z2z_xent_step(*args, s["w"], s["loss"], s["lse"], case["accumulate"], s["gh"], s["gWU"], s["gUh"], s["scratch"])
    else:
        zb.z2z_xent_loss(*args, s["loss"], s["lse"], s["scratch"])
        if case["mode"] == "autograd":
            zb.z2z_xent_grad(*args, s["lse"], s["w"], case["accumulate"], s["gh"], s["gWU"], s["gUh"], s["scratch"])
    out = {"loss": s["loss"], "lse": s["lse"]}
    return out if case["mode"] == "loss" else dict(out, hidden=s["gh"], WU=s["gWU"], Uh=s["gUh"])


def _own_clip(s, case):
    from paper_2506_01084_b200 import binding as zb
    zb.z2z_grad_clip(s["list"], case["scale"], MAX_NORM, s["norm"], s["scratch"])
    return {"norm": s["norm"], "out": s["out"]}


def _plain_xent(s, case):
    """The joint logits in fp32; a sequence's hypertokens at the rows of that sequence."""
    N, V, cap, B = case["N"], case["V"], case["cap"], case["B"]
    h, W, seq = s["hidden"].float(), s["WU"].float(), s["seq"].long()
    n = torch.tensor(s["counts"], device=DEV)
    sees = n[seq] if s["sees"] is None else s["sees"].long()
    of = [(seq == b).nonzero()[:, 0] for b in range(B)]
    l = torch.full((N, V + cap), -math.inf, device=DEV)
    l[:, :V] = h @ W.T
    for b in range(B):
        k = s["counts"][b]
        l[of[b], V:V + k] = h[of[b]] @ s["Uh"][b, :k].float().T
    seen = torch.arange(V + cap, device=DEV)[None, :] < (V + sees)[:, None]
    l = torch.where(seen, l, torch.full((), -math.inf, device=DEV))
    m = l.amax(1, keepdim=True)
    p = torch.exp(l - m)
    tot = p.sum(1, keepdim=True)
    at = s["target"].long().clamp(min=0)[:, None]
    counted = s["target"] >= 0
    lse = (m + torch.log(tot))[:, 0]
    # (differences to the maximum: the loss of a row that knows its target is small beside both)
    loss = (torch.log(tot) - (l.gather(1, at) - m))[:, 0]
    zero = torch.zeros_like(lse)
    out = {"loss": torch.where(counted, loss, zero), "lse": torch.where(counted, lse, zero)}
    if case["mode"] == "loss":
        return out
    del l
    p /= tot
    p.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    p *= torch.where(counted, s["w"], zero)[:, None]
    gh = p[:, :V] @ W
    gW, gU = s["gWU"], s["gUh"]
    t = p[:, :V].T @ h
    gW.copy_(t + gW.float() if case["accumulate"] else t)
    for b in range(B):
        k = s["counts"][b]
        q = p[of[b], V:V + k]
        gh[of[b]] += q @ s["Uh"][b, :k].float()
        t = q.T @ h[of[b]]
        gU[b, :k] = t + gU[b, :k].float() if case["accumulate"] else t
    return dict(out, hidden=gh.to(s["hidden"].dtype), WU=gW, Uh=gU)


def _plain_clip(s, case):
    """Squares in fp32, their sum in 64 bits."""
    total = torch.stack([x.float().square().sum(dtype=torch.float64) for x in s["grads"]]).sum()
    norm = (case["scale"] * torch.sqrt(total)).float()
    factor = case["scale"] * torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    for x, y in zip(s["grads"], s["outs"]):
        y.copy_(x.float() * factor)
    return {"norm": norm[None], "out": s["out"]}


# ---- what a pass cannot do without -----------------------------------------------------------------------
def work(case):
    if case["op"] == "clip":
        n = sum(math.prod(x) for x in _shapes(case))
        # in place and below the largest norm: nothing to write
        wrote = 0 if case["out"] == "same" and case["norm"] < MAX_NORM and case["scale"] == 1.0 else n
        out = case["dtype"] if case["out"] == "same" else case["out"]
        # (norm first: what the caches do not hold is read again)
        return {"bytes": n * _size(case["dtype"]) + wrote * _size(out), "flops": 2 * n + wrote}
    V, d, e = case["V"], case["d"], _size(case["dtype"])
    seq, sees, counted = _rows(case)
    live, counts = int(counted.sum()), _counts(case)
    rows = V + sum(counts)
    cols = live * V + int(sees[counted].sum())
    units = 1 if case["mode"] == "loss" else 3
    size = (rows + live) * d * e + case["N"] * 20
    if case["mode"] != "loss":
        size += case["N"] * d * e + rows * d * _size(case["grads"]) * (2 if case["accumulate"] else 1)
    return {"bytes": size, "flops": units * 2 * cols * d}


# ---- 64-bit values ---------------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_clip(s, case) if case["op"] == "clip" else _exact_xent(s, case)


def _exact_xent(s, case):
    """Sequence by sequence over the matrix that its rows meet, by log-softmax."""
    N, V, d, B, mode = case["N"], case["V"], case["d"], case["B"], case["mode"]
    W = s["WU"].double()
    loss, lse = torch.zeros(2, N, dtype=torch.float64, device=DEV).unbind(0)
    if mode != "loss":
        gh = torch.zeros(N, d, dtype=torch.float64, device=DEV)
        gW = s["gWU"].double() if case["accumulate"] else torch.zeros(V, d, dtype=torch.float64, device=DEV)
        gU = s["gUh"].double()
        if not case["accumulate"]:
            for b in range(B):
                gU[b, :s["counts"][b]] = 0.0
    for b in range(B):
        rows = ((s["seq"] == b) & s["counted"]).nonzero()[:, 0]
        for rows in rows.split(512):
            if not rows.numel():
                continue
            k = s["counts"][b]
            U = s["Uh"][b, :k].double()
            h = s["hidden"][rows].double()
            l = torch.cat([h @ W.T, h @ U.T], 1)
            if s["sees"] is not None:
                l.masked_fill_(torch.arange(V + k, device=DEV)[None, :] >= V + s["sees"][rows].long()[:, None], -math.inf)
            lp = torch.log_softmax(l, 1)
            t = s["target"][rows].long()[:, None]
            lse[rows] = torch.logsumexp(l, 1)
            loss[rows] = -lp.gather(1, t)[:, 0]
            if mode == "loss":
                continue
            q = lp.exp()
            q.scatter_add_(1, t, torch.full(t.shape, -1.0, dtype=torch.float64, device=DEV))
            q *= s["w"][rows].double()[:, None]
            gh[rows] = q[:, :V] @ W + q[:, V:] @ U
            gW.addmm_(q[:, :V].T, h)
            gU[b, :k] += q[:, V:].T @ h
    out = {"loss": loss, "lse": lse}
    return out if mode == "loss" else dict(out, hidden=gh, WU=gW, Uh=gU)


def _exact_clip(s, case):
    norm = case["scale"] * math.sqrt(math.fsum(float(torch.linalg.vector_norm(x.reshape(-1), dtype=torch.float64)) ** 2 for x in s["grads"]))
    factor = case["scale"] * min(1.0, MAX_NORM / (norm + 1e-6))
    grads = [x.double() for x in s["grads"]]
    out = s["out"].double()
    for x, y in zip(grads, _pieces(out, case)):
        torch.mul(x, factor, out=y)
    return {"norm": torch.tensor([norm], dtype=torch.float64, device=DEV), "out": out}
