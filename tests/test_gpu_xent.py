"""Cross entropy over the joint vocabulary and its gradients, against the definition in fp64."""
import numpy as np
import pytest
import torch

from oracle import xent as ox
from paper_2506_01084_b200 import binding as zb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24                # half a step of fp32
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def session(V, d, cap, B, dtype, counts):
    """A session whose sequence b has counts[b] hypertokens (prompts of distinct tokens: every pair is an entry)."""
    cb = zb.Codebook(zb.make_config(V, d, 3, cap, B, dtype, 0, 1, 8), DEV)
    lens = [c + 1 if c > 0 else 0 for c in counts]
    if max(lens) > 0:
        tokens = ((torch.arange(max(lens), device=DEV)[None, :] + torch.arange(B, device=DEV)[:, None]) % V).int().contiguous()
        codes = torch.empty_like(tokens)
        zb.z2z_lzw_encode(cb, tokens, torch.tensor(lens, dtype=torch.int32, device=DEV), codes, torch.empty(B, dtype=torch.int32, device=DEV))
    assert zb.z2z_status(cb)[1].tolist() == list(counts)
    return cb


class Case:
    def __init__(self, dtype="bf16", V=300, d=64, B=3, cap=40, counts=None, N=50, order="sequences", causal=False, skip=0.0, weights="mean",
                 grads=None, accumulate=False, scratch="most", seed=0, sharp=6.0):
        g = torch.Generator().manual_seed(seed)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.gt = {None: self.dt, "fp32": torch.float32, "bf16": torch.bfloat16}[grads]
        self.accumulate = accumulate
        counts = [min(cap, int(cap * f)) for f in np.linspace(0.3, 1.0, B)] if counts is None else counts
        self.cb = session(V, d, cap, B, dtype, counts)
        r = torch.arange(N)
        self.seq = {"sequences": r * B // max(N, 1), "turns": r % B, "random": torch.randint(0, B, (N,), generator=g)}[order]
        n = torch.tensor(counts)[self.seq]
        self.nvis = (torch.rand(N, generator=g) * (n + 1)).long() if causal else None
        sees = n if self.nvis is None else self.nvis
        self.target = (torch.rand(N, generator=g) * (V + sees)).long()
        hyper = (torch.rand(N, generator=g) < 0.4) & (sees > 0)
        self.target = torch.where(hyper, V + (torch.rand(N, generator=g) * sees).long(), self.target)
        std = 1.3 / d ** 0.5
        self.WU, self.Uh = ((torch.randn(*s, generator=g) * std).to(self.dt) for s in ((V, d), (B, cap, d)))
        row = torch.where((self.target >= V)[:, None], self.Uh[self.seq, (self.target - V).clamp(0, max(cap - 1, 0))] if cap else self.WU[0][None],
                          self.WU[self.target.clamp(max=V - 1)]).float()
        self.hidden = (torch.randn(N, d, generator=g) + sharp * torch.rand(N, 1, generator=g) * row).to(self.dt)
        if skip:
            self.target[torch.rand(N, generator=g) < skip] = -1
        self.w = {"mean": torch.full((N,), 1.0 / max(N, 1)), "none": None, "mixed": torch.rand(N, generator=g) - 0.3}[weights]
        if weights == "mixed":
            self.w[::7] = 0.0
        # (what lies behind a sequence's hypertokens is not read)
        self.g_Uh = self.Uh.clone()
        for b, c in enumerate(counts):
            self.g_Uh[b, c:] = float("nan")
        self.counts, self.V, self.d, self.N, self.B, self.cap = counts, V, d, N, B, cap
        self.gWU0, self.gUh0 = ((torch.randn(*s, generator=g) * 0.01).to(self.gt) for s in ((V, d), (B, cap, d)))
        sizes = zb.z2z_xent_scratch_bytes(self.cb.cfg, N, self.gt)
        assert sizes[0] <= sizes[1]
        size = {"least": sizes[0], "between": (sizes[0] + sizes[1]) // 2, "most": sizes[1]}[scratch]
        self.scratch = torch.full((size,), 255, dtype=torch.uint8, device=DEV)         # (NaN wherever it is read as a number)

    def dev(self, t, dtype=None):
        return None if t is None else (t if dtype is None else t.to(dtype)).to(DEV).contiguous()

    def inputs(self):
        return (self.cb, self.dev(self.hidden), self.dev(self.seq, torch.int32), self.dev(self.nvis, torch.int32), self.dev(self.WU),
                self.dev(self.g_Uh), self.dev(self.target, torch.int32))

    def run(self, mode="step"):
        N = self.N
        loss, lse = torch.full((2, N), 7.0, device=DEV).unbind(0)
        gh = torch.full((N, self.d), 7.0, dtype=self.dt, device=DEV)
        gW, gU = self.dev(self.gWU0), self.dev(self.gUh0)
        args, w = self.inputs(), self.dev(self.w)
        if mode == "step":
            zb.z2z_xent_step(*args, w, loss, lse, self.accumulate, gh, gW, gU, self.scratch)
        else:
            # (the losses alone need less)
            zb.z2z_xent_loss(*args, loss, lse, torch.full((zb.z2z_xent_scratch_bytes(self.cb.cfg, N)[N % 2],), 255, dtype=torch.uint8, device=DEV))
            zb.z2z_xent_grad(*args, lse, w, self.accumulate, gh, gW, gU, self.scratch)
        return {"loss": loss, "lse": lse, "hidden": gh, "WU": gW, "Uh": gU}

    def oracle(self):
        f = lambda t: t.double().numpy()  # noqa: E731
        return ox.cross_entropy(f(self.hidden), self.seq.numpy(), None if self.nvis is None else self.nvis.numpy(), f(self.WU), f(self.Uh),
                                self.counts, self.target.numpy(), None if self.w is None else f(self.w))

    def check(self, got, want=None):
        """Bounds.  A logit is a sum of d products: d + 8 additions in fp32 that may truncate (a step, 2 U32, each) over a
        sum of magnitudes `size`; in an fp32 session an operand's three parts hold it to 2^-24 and the products that
        are left out are below 3 x 2^-24.  An exponential then is off by the errors of its logit and of lse, by lse's own
        rounding and by ex2's few steps; a step that keeps its logits has them in steps of 2^-11; g's rounding is half a
        step of bf16, or of 24 bits.  The contracted sums add an
        error per addition over the sum of magnitudes, and the stored value its own half step."""
        want = self.oracle() if want is None else want
        live = want["live"]
        size = want["size"].max(initial=0.0)
        e_l = ((self.d + 8) * 2 * U32 + 8 * U32) * size
        e_lse = e_l + 2 * U32 * np.abs(want["lse"]).max(initial=0.0) + (64 + self.V / 64) * U32 + 2.0 ** -21
        for k in ("loss", "lse"):
            x = got[k].double().cpu().numpy()
            assert np.all(x[~live] == 0.0), k
            off = np.abs(x - want[k])
            assert np.all(off <= (2 if k == "loss" else 1) * e_lse), (k, off.max(), e_lse)
        g_step = 2.0 ** -8 if self.gt == self.dt == torch.bfloat16 else 2.0 ** -23
        rel = e_l + e_lse + 2.0 ** -20 + (2.0 ** -12 if self.gt == self.dt == torch.bfloat16 else 0.0)
        for k, dt in (("hidden", self.dt), ("WU", self.gt), ("Uh", self.gt)):
            x, y, mag = got[k].double().cpu().numpy(), want[k], want["abs_" + k]
            step = 2.0 ** -8 if k == "hidden" and self.dt == torch.bfloat16 else g_step
            terms = self.V + self.cap if k == "hidden" else self.N
            old = np.zeros_like(y)
            if k != "hidden":
                before = (self.gWU0 if k == "WU" else self.gUh0).double().numpy()
                if self.accumulate:
                    old = before
                if k == "Uh":
                    for b, c in enumerate(self.counts):
                        assert np.array_equal(x[b, c:], before[b, c:]), "rows behind a sequence's hypertokens"
                        x[b, c:] = y[b, c:] = old[b, c:] = 0.0
            tol = (step + rel + (terms + 16) * 2 * U32) * mag + STEP[dt] * (np.abs(y + old) + step * mag) * 1.01 + 1e-30
            off = np.abs(x - (y + old))
            assert np.all(off <= tol), (k, off.max(), np.max(off / tol))
            if k == "hidden":
                assert np.all(x[~live] == 0.0)


@pytest.mark.parametrize("V,d,N", [(300, 64, 50), (1, 8, 1), (257, 72, 33), (1000, 200, 300), (2500, 136, 257), (700, 520, 600)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_sizes(dtype, V, d, N):
    c = Case(dtype, V=V, d=d, N=N, cap=min(40, V - 1) if V > 1 else 0, skip=0.1, causal=True, seed=V)
    c.check(c.run())


@pytest.mark.parametrize("order", ["sequences", "turns", "random"])
@pytest.mark.parametrize("grads", [None, "fp32"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_orders_and_types(order, grads, accumulate):
    c = Case("bf16", V=900, d=96, B=7, cap=300, N=333, order=order, grads=grads, accumulate=accumulate, causal=order != "turns", skip=0.3,
             weights="mixed", seed=4)
    want = c.oracle()
    c.check(c.run("step"), want)
    c.check(c.run("autograd"), want)


def test_an_fp32_session_with_bf16_gradients_of_the_tables():
    c = Case("fp32", V=700, d=96, B=4, cap=60, N=120, grads="bf16", accumulate=True, causal=True, seed=6)
    c.check(c.run())


@pytest.mark.parametrize("scratch", ["least", "between", "most"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pieces(scratch, dtype):
    """More than one piece of the vocabulary, the last one short."""
    c = Case(dtype, V=2 * 8192 + 300 if scratch == "most" and dtype == "bf16" else 4500, d=40, B=2, cap=30, N=70, scratch=scratch, seed=9, accumulate=True)
    c.check(c.run())


@pytest.mark.parametrize("counts", [[0, 0, 0], [40, 0, 1], [16, 17, 15], [40, 40, 40]])
def test_hypertoken_counts(counts):
    c = Case("bf16", V=200, d=64, counts=counts, N=90, weights="none", seed=sum(counts))
    c.check(c.run())


def test_more_sequences_than_rows_and_long_sequences():
    c = Case("bf16", V=150, d=64, B=40, cap=20, N=9, order="random", seed=2)
    c.check(c.run())
    c = Case("bf16", V=600, d=64, B=2, cap=520, counts=[513, 300], N=700, causal=True, seed=3)
    c.check(c.run())


def test_rows_that_take_no_part_may_hold_anything():
    """NaN in hidden rows without a target, of no sequence, with an unseen target, or without weight."""
    for dtype, scratch in (("bf16", "most"), ("bf16", "least"), ("fp32", "most")):
        c = Case(dtype, V=400, d=72, B=3, cap=40, N=150, scratch=scratch, weights="mixed", causal=True, seed=8)
        none, away, unseen, light = (torch.arange(i, 150, 11) for i in range(4))
        c.target[none] = -1
        c.seq = c.seq.clone()
        c.seq[away] = torch.tensor([-1, 3, 1 << 30])[torch.arange(len(away)) % 3]
        c.target[unseen] = torch.where(torch.arange(len(unseen)) % 2 == 0, 400 + c.nvis[unseen], torch.tensor(-5))
        c.w = c.w.abs() + 0.1
        c.w[light] = 0.0
        clean = c.hidden.clone()
        bad = torch.cat([none, away, unseen])
        c.hidden[bad] = float("nan")
        want = None
        for mode in ("step", "autograd"):
            got = c.run(mode)
            st = zb.z2z_status(c.cb)[0].tolist()
            hit = {int(c.seq[r]) for r in unseen}
            assert all(bool(v & zb.ST_BAD_TOKEN) == (b in hit) for b, v in enumerate(st))
            keep, c.hidden = c.hidden, clean
            want = c.oracle() if want is None else want
            c.check(got, want)
            c.hidden = keep
        # without weight: a NaN loss, but no gradient
        c.hidden[light] = float("nan")
        got = c.run("step")
        assert bool(got["loss"][light].isnan().all()) and bool(got["lse"][light].isnan().all())
        for k in ("loss", "lse"):
            got[k][light] = torch.from_numpy(want[k]).float().to(DEV)[light]
        c.check(got, want)


def test_a_row_of_nan_reaches_its_own_gradients():
    c = Case("bf16", V=300, d=64, B=2, cap=20, N=40, weights="none", seed=1)
    c.hidden[3, 5] = float("nan")
    for mode in ("step", "autograd"):
        got = c.run(mode)
        assert bool(got["loss"][3].isnan()) and bool(got["lse"][3].isnan()) and bool(got["hidden"][3].isnan().all()) and bool(got["WU"].isnan().all())
        assert int(got["loss"].isnan().sum()) == 1 and int(got["hidden"].isnan().any(1).sum()) == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_logits_far_from_zero(dtype):
    """Rows whose logits lie hundreds apart: only differences count."""
    c = Case(dtype, V=500, d=64, B=2, cap=20, N=60, seed=12, sharp=0.0)
    c.hidden = (c.hidden.float() * torch.logspace(-1, 2.3, 60)[:, None]).to(c.dt)
    c.check(c.run("step"))
    c.check(c.run("autograd"))


def test_as_many_sequences_as_a_session_may_have():
    c = Case("bf16", V=300, d=40, B=1024, cap=9, counts=[b % 10 for b in range(1024)], N=1500, order="random", seed=15)
    c.check(c.run("step"))
    c = Case("fp32", V=300, d=40, B=1024, cap=9, counts=[b % 10 for b in range(1024)], N=1500, order="turns", skip=0.5, seed=16)
    c.check(c.run("autograd"))


def test_rows_that_belong_to_sequences_in_order():
    """Without row_seq: row r belongs to sequence r."""
    c = Case("bf16", V=900, d=64, B=70, cap=20, N=70, seed=17)
    assert torch.equal(c.seq, torch.arange(70))
    args, want = list(c.inputs()), c.oracle()
    args[2] = None
    loss, lse = torch.empty(2, 70, device=DEV).unbind(0)
    gh, gW, gU = torch.empty(70, 64, dtype=c.dt, device=DEV), c.dev(c.gWU0), c.dev(c.gUh0)
    zb.z2z_xent_step(*args, c.dev(c.w), loss, lse, False, gh, gW, gU, c.scratch)
    c.check({"loss": loss, "lse": lse, "hidden": gh, "WU": gW, "Uh": gU}, want)


def test_more_rows_than_partial_sums_are_held_for():
    """Losses of more than 8192 rows, in two shares, and pieces of the least scratch."""
    c = Case("bf16", V=70, d=16, B=3, cap=12, N=8192 + 300, order="turns", skip=0.2, scratch="least", seed=18)
    c.check(c.run("autograd"))


def test_offsets_that_pass_32_bits():
    """A table and a gradient of more than 2^31 elements: losses, and the gradients at both ends."""
    V, d, N = 530000, 4096, 6
    g = torch.Generator(device=DEV).manual_seed(3)
    cb = session(V, d, 0, 1, "bf16", [0])
    W = torch.empty(V, d, dtype=torch.bfloat16, device=DEV)
    for i in range(0, V, 1 << 16):
        W[i:i + (1 << 16)] = (torch.randn(min(1 << 16, V - i), d, generator=g, device=DEV) * 0.02).bfloat16()
    hidden = torch.randn(N, d, generator=g, device=DEV).bfloat16()
    target = torch.tensor([0, V - 1, V - 2, 1 << 19, 5, V // 2], dtype=torch.int32, device=DEV)
    seq = torch.zeros(N, dtype=torch.int32, device=DEV)
    l = torch.cat([hidden.double() @ W[i:i + (1 << 15)].double().T for i in range(0, V, 1 << 15)], 1)
    lse64, at = torch.logsumexp(l, 1), target.long()
    g64 = torch.exp(l - lse64[:, None])
    g64[torch.arange(N), at] -= 1.0
    loss, lse = torch.empty(2, N, device=DEV).unbind(0)
    gh, gW = torch.empty_like(hidden), torch.full_like(W, 7.0)
    scratch = torch.empty(zb.z2z_xent_scratch_bytes(cb.cfg, N, torch.bfloat16)[1], dtype=torch.uint8, device=DEV)
    zb.z2z_xent_step(cb, hidden, seq, None, W, None, target, None, loss, lse, False, gh, gW, None, scratch)
    # (bounds of Case.check: a logit's sum of magnitudes is below 130 here, d 0.02 0.8 0.8 and a few deviations)
    e_l = ((d + 8) * 2 * U32 + 8 * U32) * 130
    e_lse = e_l + 2 * U32 * float(lse64.abs().max()) + (64 + V / 64) * U32 + 2.0 ** -21
    assert float((lse.double() - lse64).abs().max()) <= e_lse
    assert float((loss.double() - (lse64 - l[torch.arange(N), at])).abs().max()) <= 2 * e_lse
    rel = 2.0 ** -8 + e_l + e_lse + 2.0 ** -20 + 2.0 ** -12 + (N + 16) * 2 * U32
    for rows in (slice(0, 600), slice((1 << 19) - 300, (1 << 19) + 300), slice(V - 600, V)):
        want, mag = g64[:, rows].T @ hidden.double(), g64[:, rows].abs().T @ hidden.double().abs()
        assert bool(((gW[rows].double() - want).abs() <= rel * mag + 1.01 * 2.0 ** -8 * (want.abs() + rel * mag) + 1e-30).all())
    want, mag = torch.zeros(2, N, d, dtype=torch.float64, device=DEV).unbind(0)
    for i in range(0, V, 1 << 15):
        w = W[i:i + (1 << 15)].double()
        want += g64[:, i:i + (1 << 15)] @ w
        mag += g64[:, i:i + (1 << 15)].abs() @ w.abs()
    rel += V * 2 * U32
    assert bool(((gh.double() - want).abs() <= rel * mag + 1.01 * 2.0 ** -8 * (want.abs() + rel * mag)).all())


def test_no_rows_and_no_live_rows():
    for N in (0, 5):
        c = Case("bf16", V=200, d=64, B=3, cap=30, N=N, seed=3)
        c.target[:] = -1
        got = c.run()
        assert not got["loss"].any() and not got["hidden"].any() and not got["WU"].any()
        for b, n in enumerate(c.counts):
            assert not got["Uh"][b, :n].any() and torch.equal(got["Uh"][b, n:], c.gUh0.to(DEV)[b, n:])
        c.accumulate = True
        got = c.run()
        assert torch.equal(got["WU"], c.gWU0.to(DEV)) and torch.equal(got["Uh"], c.gUh0.to(DEV))


def test_gradients_that_are_not_wanted():
    c = Case("bf16", V=300, d=64, B=3, cap=30, N=80, seed=5)
    full = c.run("autograd")
    args, w = c.inputs(), c.dev(c.w)
    for pick in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1), (0, 1, 1)):
        out = [torch.full_like(full[k], 7.0) if take else None for k, take in zip(("hidden", "WU", "Uh"), pick)]
        scratch = torch.full((zb.z2z_xent_scratch_bytes(c.cb.cfg, 80, torch.bfloat16)[1],), 255, dtype=torch.uint8, device=DEV)
        zb.z2z_xent_grad(*args, full["lse"], w, False, *out, scratch)
        for k, o in zip(("hidden", "WU", "Uh"), out):
            if o is not None and k != "Uh":
                assert torch.equal(o, full[k])
            elif o is not None:
                assert all(torch.equal(o[b, :n], full[k][b, :n]) for b, n in enumerate(c.counts))


@pytest.mark.parametrize("grads", [None, "fp32"])
def test_the_same_call_gives_the_same_bits_and_may_be_captured(grads):
    c = Case("bf16", V=3000, d=136, B=5, cap=100, N=500, order="random", skip=0.2, grads=grads, seed=7)
    want = c.run()
    for _ in range(3):
        got = c.run()
        assert all(torch.equal(got[k], want[k]) for k in got)
    args, w = c.inputs(), c.dev(c.w)
    out = {k: torch.empty_like(v) for k, v in want.items()}
    call = lambda: zb.z2z_xent_step(*args, w, out["loss"], out["lse"], False, out["hidden"], out["WU"], out["Uh"], c.scratch)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(2):
        for v in out.values():
            v.fill_(3.0)
        graph.replay()
        for k in want:
            if k != "Uh":
                assert torch.equal(out[k], want[k]), k
        assert all(torch.equal(out["Uh"][b, :n], want["Uh"][b, :n]) for b, n in enumerate(c.counts))


def test_two_streams_at_once():
    cases = [Case("bf16", V=5000, d=136, B=4, cap=100, N=300, seed=s) for s in (1, 2)]
    want = [c.run() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            got.append(c.run())
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(a[k], b[k]) for k in a)


def test_gradients_against_differences():
    """The gradient along a direction against the losses' differences (fp32: what differences can resolve)."""
    c = Case("fp32", V=120, d=32, B=2, cap=16, N=40, weights="mixed", causal=True, seed=21)
    got = c.run()
    g = torch.Generator().manual_seed(1)
    h = 2.0 ** -6
    for k, t in (("hidden", c.hidden), ("WU", c.WU), ("g_Uh", c.g_Uh)):
        step = torch.randn(t.shape, generator=g)
        base, sums = t.clone(), []
        for sign in (1, -1):
            t.copy_(base + sign * h * step)
            sums.append(float((c.run()["loss"].double().cpu() * c.w.double()).sum()))
        t.copy_(base)
        grad = got["Uh" if k == "g_Uh" else k].double().cpu()
        dots = (grad * step.double())
        along = float(dots[~base.isnan()].sum()) if k != "g_Uh" else sum(float(dots[b, :n].sum()) for b, n in enumerate(c.counts))
        diff = (sums[0] - sums[1]) / (2 * h)
        # third derivatives of a log-sum-exp are below 2 max |dl|^3; the losses' rounding over 2 h
        dl = 6.0 * c.d ** 0.5
        assert abs(diff - along) <= h * h / 6 * 2 * dl ** 3 * float(c.w.abs().sum()) + 40 * 2.0 ** -20 / h, (k, diff, along)
