"""Arguments that the embedding, distillation and beam calls refuse on the host.  Every call here is refused before
anything is enqueued, so that no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2506_01084_b200 import binding as zb

P, I64, F = C.c_void_p, C.c_int64, C.c_float
HERE = 4096                     # an address that is never used: the calls are refused before
V, D, M, CAP, B = 100, 16, 3, 8, 6


@pytest.fixture(scope="module")
def cb():
    """A handle.  Without a GPU its session cannot be started, which leaves the configuration that the checks go by."""
    if torch.cuda.is_available():
        pytest.skip("the addresses here are made up: a call that was not refused must find no GPU")
    cfg = zb.make_config(V, D, M, CAP, B, "bf16", 0, 1, 8)
    h = P(0)
    assert zb.lib().z2z_codebook_init(C.byref(h), C.byref(cfg), P(1 << 20), C.c_size_t(1 << 40), None) == -3 and h.value
    yield h
    zb.lib().z2z_codebook_destroy(h)


def refused(rc, text, code=-1):
    assert rc == code
    assert text in zb.lib().z2z_last_error().decode()


def test_embed_lookup_scaled(cb):
    f = zb.lib().z2z_embed_lookup_scaled
    refused(f(None, HERE, 1, None, HERE, HERE, 1.0, HERE, None), "cb is NULL")
    refused(f(cb, HERE, -1, None, HERE, HERE, 1.0, HERE, None), "N < 0")
    for bad in (float("nan"), float("inf")):
        refused(f(cb, HERE, 1, None, HERE, HERE, bad, HERE, None), "scale")
    refused(f(cb, None, 1, None, HERE, HERE, 1.0, HERE, None), "NULL")
    refused(f(cb, HERE, 1, None, HERE, None, 1.0, HERE, None), "d_Eh is NULL")
    refused(f(cb, HERE, 1, None, HERE + 8, HERE, 1.0, HERE, None), "aligned")
    refused(f(cb, HERE, 1, None, HERE, HERE, 1.0, HERE + 2, None), "aligned")
    refused(f(cb, HERE, B + 1, None, HERE, HERE, 1.0, HERE, None), "d_row_seq")
    assert f(cb, None, 0, None, None, None, 1.0, None, None) == 0


def test_embed_grad(cb):
    f = zb.lib().z2z_embed_grad
    cfg = zb.make_config(V, D, M, CAP, B, "bf16", 0, 1, 8)
    need = zb.z2z_embed_grad_scratch_bytes(cfg, 4)
    ok = dict(codes=HERE, N=4, seq=None, g=HERE, scale=1.0, dt=0, acc=1, gW=HERE, gE=HERE, scr=HERE, by=need)

    def call(**kw):
        a = dict(ok, **kw)
        return f(cb, a["codes"], a["N"], a["seq"], a["g"], a["scale"], a["dt"], a["acc"], a["gW"], a["gE"], a["scr"], a["by"], None)

    refused(call(N=-1), "N")
    refused(call(N=(1 << 24) + 1), "2^24")
    refused(call(scale=float("nan")), "scale")
    refused(call(dt=7), "grad_dtype")
    refused(call(acc=2), "accumulate")
    refused(call(gW=None, gE=None), "both NULL")
    refused(call(codes=None), "NULL")
    refused(call(g=None), "NULL")
    refused(call(gW=HERE + 4), "aligned")
    refused(call(g=HERE + 2), "aligned")
    refused(call(N=B + 1), "d_row_seq")
    refused(call(scr=None), "scratch")
    refused(call(scr=HERE + 16), "scratch")
    refused(call(by=need - 1), "scratch", -2)
    refused(f(None, HERE, 1, None, HERE, 1.0, 0, 1, HERE, HERE, HERE, need, None), "cb is NULL")
    assert call(N=0, by=0, scr=None, codes=None, g=None) == 0                    # nothing to add
    with pytest.raises(zb.Z2ZError):
        zb.z2z_embed_grad_scratch_bytes(cfg, -1)
    with pytest.raises(zb.Z2ZError):
        zb.z2z_embed_grad_scratch_bytes(zb.make_config(V, 12, M, CAP, B, "bf16", 0, 1, 8), 1)
    big, small = (zb.z2z_embed_grad_scratch_bytes(cfg, n) for n in (1 << 24, 1))
    assert big > small > 0


def test_distill(cb):
    lib = zb.lib()
    ok = dict(l=HERE, dt=0, N=2, cols=10, ld=10, n=None, ids=HERE, t=HERE, K=3, T=1.0)

    def fwd(loss=HERE, lse=HERE, grad=None, **kw):
        a = dict(ok, **kw)
        return lib.z2z_distill_loss(a["l"], a["dt"], a["N"], a["cols"], a["ld"], a["n"], a["ids"], a["t"], a["K"], a["T"], None, loss, lse, grad, None)

    def bwd(lse=HERE, gl=HERE, grad=HERE, **kw):
        a = dict(ok, **kw)
        return lib.z2z_distill_grad(a["l"], a["dt"], a["N"], a["cols"], a["ld"], a["n"], a["ids"], a["t"], a["K"], a["T"], lse, gl, grad, None)

    for f in (fwd, bwd):
        refused(f(dt=2), "dtype")
        refused(f(N=-1), "N < 0")
        refused(f(cols=0), "cols")
        refused(f(cols=(1 << 24) + 1, ld=1 << 25), "cols")
        refused(f(ld=9), "ld")
        refused(f(K=-1), "K")
        refused(f(K=1025), "K")
        for T in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
            refused(f(T=T), "temperature")
        refused(f(l=None), "d_logits")
        refused(f(l=HERE + 2), "aligned")
        refused(f(dt=1, l=HERE + 1), "aligned")
        refused(f(ids=None), "teacher")
        refused(f(t=None), "teacher")
        assert f(N=0) == 0
    refused(fwd(loss=None), "d_loss")
    refused(fwd(lse=None), "d_lse")
    refused(fwd(grad=HERE + 2), "aligned")
    refused(bwd(lse=None), "d_lse")
    refused(bwd(gl=None), "d_grad_loss")
    refused(bwd(grad=None), "d_grad")


def test_beam_select(cb):
    f = zb.lib().z2z_beam_select
    ok = dict(beams=3, l=HERE, lse=HERE, s=HERE, fin=None, eos=-1, p=HERE, c=HERE, ns=HERE)

    def call(**kw):
        a = dict(ok, **kw)
        return f(cb, a["beams"], a["l"], a["lse"], a["s"], a["fin"], a["eos"], a["p"], a["c"], a["ns"], None, None, None)

    for w in (0, -1, 33):
        refused(call(beams=w), "beams")
    refused(call(beams=4), "multiple")                       # B = 6
    refused(call(eos=-2), "eos")
    refused(call(eos=V), "eos")
    for k in ("l", "lse", "s", "p", "c", "ns"):
        refused(call(**{k: None}), "NULL")
    refused(call(l=HERE + 2), "aligned")
    refused(f(None, 3, HERE, HERE, HERE, None, -1, HERE, HERE, HERE, None, None, None), "cb is NULL")


def test_beam_reorder(cb):
    f = zb.lib().z2z_beam_reorder
    rows = (zb.SeqRows * 1)(zb.SeqRows(HERE, 64, 64))

    def call(p=HERE, E=HERE, U=HERE, ef=None, st=rows, n=1):
        return f(cb, p, E, U, ef, None, st, n, None)

    refused(f(None, HERE, HERE, HERE, None, None, None, 0, None), "cb is NULL")
    refused(call(p=None), "d_parent")
    refused(call(E=None), "d_Eh / d_Uh")
    refused(call(U=None), "d_Eh / d_Uh")
    refused(call(E=HERE + 8), "aligned")
    refused(call(ef=HERE + 4), "aligned")
    refused(call(n=9), "n_states")
    refused(call(n=-1), "n_states")
    refused(call(st=None), "h_states")
    for bad in ((None, 64, 64), (HERE + 2, 64, 64), (HERE, 64, 62), (HERE, 66, 64), (HERE, 60, 64)):
        refused(call(st=(zb.SeqRows * 1)(zb.SeqRows(*bad))), "state")


def test_the_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros(4, 8)
    with pytest.raises(zb.Z2ZError):                         # host memory
        zb.z2z_distill_loss(x, None, None, None, 1.0, None, torch.zeros(4), torch.zeros(4))
    with pytest.raises(zb.Z2ZError):
        zb.z2z_distill_loss(x.half(), None, None, None, 1.0, None, torch.zeros(4), torch.zeros(4))
