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
        size = sizes[0 if scratch == "least" else 1]
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
        rounding and by ex2's few steps; g's rounding is half a step of bf16, or of 24 bits.  The contracted sums add an
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
        rel = e_l + e_lse + 2.0 ** -20
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


@pytest.mark.parametrize("scratch", ["least", "most"])
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
