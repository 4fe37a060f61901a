"""Arguments that the cross entropy and the gradient clipping refuse on the host.  Every call here is refused before
anything is enqueued, so that no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2506_01084_b200 import binding as zb

HERE = 4096                     # an address that is never used: the calls are refused before
V, D, M, CAP, B = 100, 16, 3, 8, 6
CFG = zb.make_config(V, D, M, CAP, B, "bf16", 0, 1, 8)


@pytest.fixture(scope="module")
def cb():
    """A handle.  Without a GPU its session cannot be started, which leaves the configuration that the checks go by."""
    if torch.cuda.is_available():
        pytest.skip("the addresses here are made up: a call that was not refused must find no GPU")
    h = C.c_void_p(0)
    assert zb.lib().z2z_codebook_init(C.byref(h), C.byref(CFG), C.c_void_p(1 << 20), C.c_size_t(1 << 40), None) == -3 and h.value
    yield h
    zb.lib().z2z_codebook_destroy(h)


def refused(rc, text, code=-1):
    assert rc == code
    assert text in zb.lib().z2z_last_error().decode()


def test_xent(cb):
    lib = zb.lib()
    least = zb.z2z_xent_scratch_bytes(CFG, 4, torch.float32)[0]
    least_loss = zb.z2z_xent_scratch_bytes(CFG, 4)[0]
    assert 0 < least_loss < least
    ok = dict(cb=cb, h=HERE, N=4, seq=None, nvis=None, W=HERE, U=HERE, t=HERE, loss=HERE, lse=HERE, w=None, dt=0, acc=1, gh=HERE, gW=HERE, gU=HERE,
              scr=HERE, by=least)

    def call(kind, **kw):
        a = dict(ok, **kw)
        rows = (a["cb"], a["h"], a["N"], a["seq"], a["nvis"], a["W"], a["U"], a["t"])
        grads = (a["dt"], a["acc"], a["gh"], a["gW"], a["gU"], a["scr"], a["by"], None)
        if kind == "loss":
            return lib.z2z_xent_loss(*rows, a["loss"], a["lse"], a["scr"], a["by"], None)
        if kind == "grad":
            return lib.z2z_xent_grad(*rows, a["lse"], a["w"], *grads)
        return lib.z2z_xent_step(*rows, a["w"], a["loss"], a["lse"], *grads)

    for kind in ("loss", "grad", "step"):
        refused(call(kind, cb=None), "cb is NULL")
        refused(call(kind, N=-1), "N")
        refused(call(kind, N=(1 << 20) + 1), "2^20")
        for k in ("h", "W", "t"):
            refused(call(kind, **{k: None}), "NULL")
        refused(call(kind, U=None), "d_Uh is NULL")
        for k in ("h", "W", "U"):
            refused(call(kind, **{k: HERE + 8}), "aligned")
        for k in ("t", "seq", "nvis", "lse"):
            refused(call(kind, **{k: HERE + 2}), "aligned")
        refused(call(kind, lse=None), "d_lse")
        refused(call(kind, N=B + 1, by=1 << 40), "d_row_seq")
        refused(call(kind, scr=None), "scratch")
        refused(call(kind, scr=HERE + 16), "scratch")
        refused(call(kind, by=(least_loss if kind == "loss" else least) - 1), "scratch", -2)
    for kind in ("grad", "step"):
        refused(call(kind, dt=2), "grad_dtype")
        refused(call(kind, acc=2), "accumulate")
        refused(call(kind, gh=None, gW=None, gU=None), "no gradient")
        for k in ("gh", "gW", "gU"):
            refused(call(kind, **{k: HERE + 4}), "aligned")
        refused(call(kind, w=HERE + 1), "aligned")
    for kind in ("loss", "step"):
        refused(call(kind, loss=None), "d_loss")
    assert call("loss", N=0, h=None, W=None, U=None, t=None, loss=None, lse=None, scr=None, by=0) == 0
    assert call("step", N=0, h=None, W=None, U=None, t=None, loss=None, lse=None, scr=None, by=0) == 0        # accumulates nothing


def test_xent_scratch():
    for bad in ((CFG, -1, None), (CFG, (1 << 20) + 1, None), (zb.make_config(V, 12, M, CAP, B, "bf16", 0, 1, 8), 1, None), (CFG, 1, torch.float16)):
        with pytest.raises(zb.Z2ZError):
            zb.z2z_xent_scratch_bytes(*bad)
    assert zb.lib().z2z_xent_scratch_bytes(C.byref(CFG), 1, -1, None, None) == -1
    assert zb.lib().z2z_xent_scratch_bytes(C.byref(CFG), 1, 2, C.byref(C.c_size_t()), C.byref(C.c_size_t())) == -1
    assert zb.z2z_xent_scratch_bytes(CFG, 0, torch.float32) == (0, 0)
    for cfg in (CFG, zb.make_config(128256, 4096, M, 4096, 32, "bf16", 0, 1, 8), zb.make_config(8009, 520, M, 0, 5, "fp32", 0, 1, 8)):
        for dt in (None, torch.float32, torch.bfloat16):
            last = (0, 0)
            for N in (1, 2, 33, 256, 257, 5000, 1 << 20):
                sizes = zb.z2z_xent_scratch_bytes(cfg, N, dt)
                assert 0 < sizes[0] <= sizes[1] and sizes[0] >= last[0], (N, dt, sizes)
                last = sizes


def test_grad_clip():
    if torch.cuda.is_available():
        pytest.skip("the addresses here are made up: a call that was not refused must find no GPU")
    lib = zb.lib()
    need = C.c_size_t(0)
    assert lib.z2z_grad_clip_scratch_bytes(2, C.byref(need)) == 0 and need.value > 0

    def call(recs=((HERE, HERE, 4, 0, 0), (HERE, None, 4, 1, 9)), n=None, scale=1.0, most=1.0, norm=HERE, scr=HERE, by=None):
        rec = (zb.GradTensor * max(1, len(recs)))(*[zb.GradTensor(*r) for r in recs])
        return lib.z2z_grad_clip(rec, len(recs) if n is None else n, scale, most, norm, scr, need.value if by is None else by, None)

    refused(call(n=-1), "65536")
    refused(call(n=(1 << 16) + 1), "65536")
    refused(lib.z2z_grad_clip(None, 1, 1.0, 1.0, HERE, HERE, need.value, None), "h_tensors")
    for bad in (float("nan"), float("inf")):
        refused(call(scale=bad), "scale")
    for bad in (0.0, -1.0, float("nan")):
        refused(call(most=bad), "max_norm")
    refused(call(norm=HERE + 2), "aligned")
    for rec, text in (((HERE, HERE, -1, 0, 0), "negative"), ((HERE, HERE, 4, 2, 0), "dtype"), ((HERE, HERE, 4, 0, 3), "dtype"), ((None, HERE, 4, 0, 0), "d_grad"),
                      ((HERE + 2, HERE, 4, 0, 0), "aligned"), ((HERE, HERE + 1, 4, 0, 1), "aligned"), ((HERE, HERE, 4, 0, 1), "in place"),
                      ((HERE, HERE, 1 << 44, 0, 0), "2^43")):
        refused(call(recs=[rec]), text)
    refused(call(scr=None), "scratch")
    refused(call(scr=HERE + 4), "scratch")
    refused(call(by=need.value - 1), "scratch", -2)
    assert lib.z2z_grad_clip_scratch_bytes(-1, C.byref(need)) == -1
    assert lib.z2z_grad_clip_scratch_bytes(1, None) == -1


def test_the_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros(4)
    with pytest.raises(zb.Z2ZError):                         # host memory
        zb.grad_tensors([x])
    with pytest.raises(zb.Z2ZError):
        zb.grad_tensors([x], [])
