"""ctypes binding of the C ABI in include/z2z.h: same names, argument marshalling only.

Every call takes torch tensors (device memory owned by the caller) and forwards raw pointers and
the current CUDA stream.  Nothing is computed here; if the shared library has not been built the
import of the library fails loudly (there is no fallback path).
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libz2z.so")

OK = 0
ST_CAP_FROZEN, ST_BAD_TOKEN, ST_TABLE_FULL, ST_WAIT_TIMEOUT, ST_OUTPUT_TRUNCATED, ST_HALF_RANGE = 1, 2, 4, 8, 16, 32
ST_BAD_PARENT = 64
DTYPE_FP32, DTYPE_BF16 = 0, 1
SELECT_ARGMAX, SELECT_GUMBEL = 0, 1
CODE_NONE, CODE_SELECTED = -1, -2
CACHE_EMBED, CACHE_UNEMBED = 0, 1
DECODE_RESIDENT, DECODE_REPLAY = 0, 1

EXPORTS = ["z2z_workspace_bytes", "z2z_codebook_init", "z2z_lzw_encode", "z2z_lzw_step",
           "z2z_hyper_embed", "z2z_dynamic_logits", "z2z_decode_step", "z2z_status",
           "z2z_codebook_read", "z2z_codebook_destroy", "z2z_last_error", "z2z_profile",
           "z2z_profile_read", "z2z_set_tensor_cores", "z2z_logits_static_scratch",
           "z2z_lzw_decode", "z2z_embed_lookup", "z2z_upload_rows", "z2z_sample_filtered",
           "z2z_set_encoder_half_scratch", "z2z_embed_lookup_scaled", "z2z_embed_grad_scratch_bytes", "z2z_embed_grad",
           "z2z_distill_loss", "z2z_distill_grad", "z2z_set_distill_wait_limit", "z2z_beam_select", "z2z_beam_reorder",
           "z2z_xent_scratch_bytes", "z2z_xent_loss", "z2z_xent_grad", "z2z_xent_step", "z2z_set_xent_wait_limit", "z2z_grad_clip_scratch_bytes",
           "z2z_grad_clip"]


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("V", "d", "M", "cap", "B", "dtype", "enc_layers",
                                         "enc_heads", "enc_dff", "tied")]


class EncoderWeights(C.Structure):
    _fields_ = [("tensors", C.POINTER(C.c_void_p)), ("n_tensors", C.c_int32)]


class SeqRows(C.Structure):
    _fields_ = [("d_base", C.c_void_p), ("stride", C.c_size_t), ("bytes", C.c_size_t)]


class GradTensor(C.Structure):
    _fields_ = [("d_grad", C.c_void_p), ("d_out", C.c_void_p), ("numel", C.c_int64), ("grad_dtype", C.c_int32), ("out_dtype", C.c_int32)]


_P, _I, _F, _L = C.c_void_p, C.c_int32, C.c_float, C.c_int64
# Argument types of the calls that are made with plain Python numbers (an address of 0 is None).
_ARGTYPES = {
    "z2z_embed_lookup_scaled": [_P, _P, _I, _P, _P, _P, _F, _P, _P],
    "z2z_embed_grad": [_P, _P, _I, _P, _P, _F, _I, _I, _P, _P, _P, C.c_size_t, _P],
    "z2z_distill_loss": [_P, _I, _I, _I, _L, _P, _P, _P, _I, _F, _P, _P, _P, _P, _P],
    "z2z_distill_grad": [_P, _I, _I, _I, _L, _P, _P, _P, _I, _F, _P, _P, _P, _P],
    "z2z_set_distill_wait_limit": [_L],
    "z2z_xent_scratch_bytes": [C.POINTER(Config), _I, _I, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)],
    "z2z_xent_loss": [_P, _P, _I, _P, _P, _P, _P, _P, _P, _P, _P, C.c_size_t, _P],
    "z2z_xent_grad": [_P, _P, _I, _P, _P, _P, _P, _P, _P, _P, _I, _I, _P, _P, _P, _P, C.c_size_t, _P],
    "z2z_xent_step": [_P, _P, _I, _P, _P, _P, _P, _P, _P, _P, _P, _I, _I, _P, _P, _P, _P, C.c_size_t, _P],
    "z2z_set_xent_wait_limit": [_L],
    "z2z_grad_clip_scratch_bytes": [_I, C.POINTER(C.c_size_t)],
    "z2z_grad_clip": [C.POINTER(GradTensor), _I, _F, _F, _P, _P, C.c_size_t, _P],
    "z2z_beam_select": [_P, _I, _P, _P, _P, _P, _I, _P, _P, _P, _P, _P, _P],
    "z2z_beam_reorder": [_P, _P, _P, _P, _P, _P, C.POINTER(SeqRows), _I, _P],
}


class Z2ZError(RuntimeError):
    pass


_lib = None


def lib() -> C.CDLL:
    """Load the shared library (once).  Raises if it is missing: build it first with
    ``python -m paper_2506_01084_b200.build``."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise Z2ZError(f"{LIB_PATH} not found: run `python -m paper_2506_01084_b200.build`")
        _lib = C.CDLL(LIB_PATH)
        _lib.z2z_last_error.restype = C.c_char_p
        for name in EXPORTS:
            if name != "z2z_last_error":
                getattr(_lib, name).restype = C.c_int32
        for name, types in _ARGTYPES.items():
            getattr(_lib, name).argtypes = types
    return _lib


def _check(rc: int):
    if rc != OK:
        raise Z2ZError(f"z2z error {rc}: {lib().z2z_last_error().decode()}")


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return C.c_void_p(0)
    assert t.is_contiguous(), "tensors passed to the ABI must be contiguous"
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _need(ok: bool, what: str):
    if not ok:
        raise Z2ZError(what)


def _dev(t: Optional[torch.Tensor], dtype, numel: int, name: str):
    """Address of a contiguous device tensor of this type and size, None for None."""
    if t is None:
        return None
    if t.dtype is dtype and t.numel() == numel and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    raise Z2ZError(f"{name} must be a contiguous device tensor of {numel} {dtype}")


# Handle of a device's current stream, without the Stream object that the public call makes around it (1 us of a small call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _enqueue(fn, on: torch.Tensor, *args):
    """The call on the current stream of the device that `on` lies on."""
    dev = on.get_device()
    if dev == torch.cuda.current_device():
        rc = fn(*args, _raw_stream(dev))
    elif dev < 0:
        raise Z2ZError("device tensors are needed")
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc:
        _check(rc)


def make_config(V, d, M, cap, B, dtype, enc_layers, enc_heads, enc_dff, tied=0) -> Config:
    if dtype in ("fp32", torch.float32):
        dt = DTYPE_FP32
    elif dtype in ("bf16", torch.bfloat16):
        dt = DTYPE_BF16
    else:
        dt = int(dtype)
    return Config(V, d, M, cap, B, dt, enc_layers, enc_heads, enc_dff, tied)


def encoder_weights(tensors: Sequence[torch.Tensor]) -> EncoderWeights:
    """HOST array of DEVICE pointers in ABI order.  The returned struct keeps the array alive."""
    arr = (C.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
    ew = EncoderWeights(C.cast(arr, C.POINTER(C.c_void_p)), len(tensors))
    ew._keep = (arr, list(tensors))
    return ew


def z2z_workspace_bytes(cfg: Config) -> int:
    out = C.c_size_t(0)
    _check(lib().z2z_workspace_bytes(C.byref(cfg), C.byref(out)))
    return out.value


class Codebook:
    """Owns the opaque handle; the workspace tensor is allocated by the caller side (torch)."""

    def __init__(self, cfg: Config, device="cuda:0"):
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = z2z_workspace_bytes(cfg)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        off = (-self.workspace.data_ptr()) % 256
        self._ws_ptr = self.workspace.data_ptr() + off
        self._ws_bytes = nbytes
        self.handle = C.c_void_p(0)
        z2z_codebook_init(self)

    def __del__(self):
        try:
            if self.handle and _lib is not None:
                _lib.z2z_codebook_destroy(self.handle)
                self.handle = C.c_void_p(0)
        except Exception:
            pass


def z2z_codebook_init(cb: Codebook):
    _check(lib().z2z_codebook_init(C.byref(cb.handle), C.byref(cb.cfg), C.c_void_p(cb._ws_ptr),
                                   C.c_size_t(cb._ws_bytes), _stream()))


def z2z_lzw_encode(cb: Codebook, tokens: torch.Tensor, lens: Optional[torch.Tensor],
                   codes: torch.Tensor, code_lens: torch.Tensor,
                   entries_after: Optional[torch.Tensor] = None):
    T_max = tokens.shape[1] if tokens.dim() == 2 else 0
    _check(lib().z2z_lzw_encode(cb.handle, _ptr(tokens), _ptr(lens), C.c_int32(T_max), _ptr(codes),
                                _ptr(code_lens), _ptr(entries_after), _stream()))


def z2z_lzw_step(cb: Codebook, new_codes: torch.Tensor, active: Optional[torch.Tensor],
                 new_entry: Optional[torch.Tensor]):
    _check(lib().z2z_lzw_step(cb.handle, _ptr(new_codes), _ptr(active), _ptr(new_entry), _stream()))


def z2z_hyper_embed(cb: Codebook, which: int, table: torch.Tensor, enc: EncoderWeights,
                    first: Optional[torch.Tensor], count: Optional[torch.Tensor], max_entries: int,
                    cache: torch.Tensor, cache_f32: Optional[torch.Tensor] = None):
    _check(lib().z2z_hyper_embed(cb.handle, C.c_int32(which), _ptr(table), C.byref(enc),
                                 _ptr(first), _ptr(count), C.c_int32(max_entries), _ptr(cache),
                                 _ptr(cache_f32), _stream()))


def z2z_dynamic_logits(cb: Codebook, hidden: torch.Tensor, row_seq: Optional[torch.Tensor],
                       row_nvis: Optional[torch.Tensor], W_U: torch.Tensor, U_h: torch.Tensor,
                       select: int, temperature: float, seed: int, step: int,
                       targets: Optional[torch.Tensor], lse: Optional[torch.Tensor],
                       argmax: Optional[torch.Tensor], max_logit: Optional[torch.Tensor],
                       sample: Optional[torch.Tensor] = None,
                       target_logit: Optional[torch.Tensor] = None,
                       logits_debug: Optional[torch.Tensor] = None):
    N = hidden.shape[0]
    _check(lib().z2z_dynamic_logits(cb.handle, _ptr(hidden), C.c_int32(N), _ptr(row_seq),
                                    _ptr(row_nvis), _ptr(W_U), _ptr(U_h), C.c_int32(select),
                                    C.c_float(temperature), C.c_uint64(seed), C.c_uint64(step),
                                    _ptr(targets), _ptr(lse), _ptr(argmax), _ptr(max_logit),
                                    _ptr(sample), _ptr(target_logit), _ptr(logits_debug), _stream()))


def z2z_decode_step(cb: Codebook, hidden: torch.Tensor, W_E: torch.Tensor, W_U: torch.Tensor,
                    enc_E: EncoderWeights, enc_U: EncoderWeights, E_h: torch.Tensor,
                    U_h: torch.Tensor, select: int, temperature: float, seed: int, step: int,
                    forced: Optional[torch.Tensor], next_codes: torch.Tensor,
                    selected: Optional[torch.Tensor], lse: Optional[torch.Tensor],
                    new_entry: Optional[torch.Tensor] = None,
                    E_h_f32: Optional[torch.Tensor] = None, U_h_f32: Optional[torch.Tensor] = None,
                    next_embed: Optional[torch.Tensor] = None):
    _check(lib().z2z_decode_step(cb.handle, _ptr(hidden), _ptr(W_E), _ptr(W_U), C.byref(enc_E),
                                 C.byref(enc_U), _ptr(E_h), _ptr(U_h), C.c_int32(select),
                                 C.c_float(temperature), C.c_uint64(seed), C.c_uint64(step),
                                 _ptr(forced), _ptr(next_codes), _ptr(selected), _ptr(lse),
                                 _ptr(new_entry), _ptr(E_h_f32), _ptr(U_h_f32), _ptr(next_embed), _stream()))


def z2z_lzw_decode(cb: Codebook, codes: torch.Tensor, code_lens: Optional[torch.Tensor], mode: int,
                   tokens: torch.Tensor, token_lens: torch.Tensor):
    """codes [B, Tc_max] int32 -> tokens [B, T_out_max] int32, token_lens [B] (device tensors)."""
    Tc_max = codes.shape[1] if codes.dim() == 2 else 0
    T_out = tokens.shape[1] if tokens.dim() == 2 else 0
    _check(lib().z2z_lzw_decode(cb.handle, _ptr(codes), _ptr(code_lens), C.c_int32(Tc_max),
                                C.c_int32(mode), _ptr(tokens), _ptr(token_lens), C.c_int32(T_out),
                                _stream()))


def z2z_embed_lookup(cb: Codebook, codes: torch.Tensor, row_seq: Optional[torch.Tensor],
                     W_E: torch.Tensor, E_h: torch.Tensor, out: torch.Tensor):
    """codes [N] int32 -> out [N, d]: W_E rows for base tokens, cached E_h rows for hypertokens."""
    _check(lib().z2z_embed_lookup(cb.handle, _ptr(codes), C.c_int32(codes.numel()), _ptr(row_seq),
                                  _ptr(W_E), _ptr(E_h), _ptr(out), _stream()))


def _table_dtype(cb: Codebook):
    return torch.bfloat16 if cb.cfg.dtype == DTYPE_BF16 else torch.float32


def _cache(cb: Codebook, t: Optional[torch.Tensor], dtype, name: str):
    """Address of a [B, cap, d] tensor; sessions without hypertokens have none."""
    return _dev(t, dtype, cb.cfg.B * cb.cfg.cap * cb.cfg.d, name) if cb.cfg.cap > 0 else None


def z2z_embed_lookup_scaled(cb: Codebook, codes: torch.Tensor, row_seq: Optional[torch.Tensor], W_E: torch.Tensor,
                            E_h: Optional[torch.Tensor], scale: float, out: torch.Tensor):
    """codes [N] int32 -> out [N, d] = scale * row: W_E rows for base tokens, cached E_h rows for hypertokens."""
    c, N, dt = cb.cfg, codes.numel(), _table_dtype(cb)
    _enqueue(lib().z2z_embed_lookup_scaled, out, cb.handle, _dev(codes, torch.int32, N, "codes"), N,
             _dev(row_seq, torch.int32, N, "row_seq"), _dev(W_E, dt, c.V * c.d, "W_E"), _cache(cb, E_h, dt, "E_h"),
             scale, _dev(out, dt, N * c.d, "out"))


def z2z_embed_grad_scratch_bytes(cfg: Config, N: int) -> int:
    out = C.c_size_t(0)
    _check(lib().z2z_embed_grad_scratch_bytes(C.byref(cfg), C.c_int32(N), C.byref(out)))
    return out.value


def z2z_embed_grad(cb: Codebook, codes: torch.Tensor, row_seq: Optional[torch.Tensor], grad_out: torch.Tensor, scale: float,
                   accumulate: bool, grad_WE: Optional[torch.Tensor], grad_Eh: Optional[torch.Tensor], scratch: torch.Tensor):
    """Gradient of z2z_embed_lookup_scaled for its tables (None: a frozen one), of the type the gradients have (fp32 or
    bf16, both the same); scratch: uint8 tensor of z2z_embed_grad_scratch_bytes."""
    c, N = cb.cfg, codes.numel()
    some = grad_WE if grad_WE is not None else grad_Eh
    _need(some is not None and some.dtype in (torch.float32, torch.bfloat16), "grad_WE or grad_Eh must be given, fp32 or bf16")
    _enqueue(lib().z2z_embed_grad, some, cb.handle, _dev(codes, torch.int32, N, "codes"), N, _dev(row_seq, torch.int32, N, "row_seq"),
             _dev(grad_out, _table_dtype(cb), N * c.d, "grad_out"), scale,
             DTYPE_FP32 if some.dtype == torch.float32 else DTYPE_BF16, 1 if accumulate else 0,
             _dev(grad_WE, some.dtype, c.V * c.d, "grad_WE"), _cache(cb, grad_Eh, some.dtype, "grad_Eh"),
             _dev(scratch, torch.uint8, scratch.numel(), "scratch"), scratch.numel())


def _distill_args(logits: torch.Tensor, n_cols, teacher_ids, teacher_logits, temperature: float):
    _need(logits.dim() == 2 and logits.is_cuda and logits.dtype in (torch.float32, torch.bfloat16)
          and (logits.stride(1) == 1 or logits.shape[1] == 1), "logits must be a device matrix with contiguous rows, fp32 or bf16")
    N, cols = logits.shape
    K = teacher_ids.shape[1] if teacher_ids is not None else 0
    return N, (logits.data_ptr(), DTYPE_FP32 if logits.dtype == torch.float32 else DTYPE_BF16, N, cols,
               logits.stride(0) if N > 1 else cols, _dev(n_cols, torch.int32, N, "n_cols"), _dev(teacher_ids, torch.int32, N * K, "teacher_ids"),
               _dev(teacher_logits, torch.float32, N * K, "teacher_logits"), K, temperature)


def _like(grad: Optional[torch.Tensor], logits: torch.Tensor):
    if grad is None:
        return None
    _need(grad.dtype == logits.dtype and grad.is_cuda and grad.shape == logits.shape
          and (grad.stride() == logits.stride() or grad.shape[0] == 1 and grad.is_contiguous()),
          "grad must have the shape, type and strides of logits")
    return grad.data_ptr()


def z2z_distill_loss(logits: torch.Tensor, n_cols: Optional[torch.Tensor], teacher_ids: Optional[torch.Tensor],
                     teacher_logits: Optional[torch.Tensor], temperature: float, row_weight: Optional[torch.Tensor],
                     loss: torch.Tensor, lse: torch.Tensor, grad: Optional[torch.Tensor] = None):
    """logits [N, cols] (rows may be strided), teacher_ids / teacher_logits [N, K] -> loss [N], lse [N] and, when given, the
    gradient of sum(row_weight * loss) for the logits."""
    N, args = _distill_args(logits, n_cols, teacher_ids, teacher_logits, temperature)
    _enqueue(lib().z2z_distill_loss, logits, *args, _dev(row_weight, torch.float32, N, "row_weight"),
             _dev(loss, torch.float32, N, "loss"), _dev(lse, torch.float32, N, "lse"), _like(grad, logits))


def z2z_distill_grad(logits: torch.Tensor, n_cols: Optional[torch.Tensor], teacher_ids: Optional[torch.Tensor],
                     teacher_logits: Optional[torch.Tensor], temperature: float, lse: torch.Tensor, grad_loss: torch.Tensor,
                     grad: torch.Tensor):
    """Backward pass of z2z_distill_loss: lse as it left it, grad_loss [N] -> grad [N, cols]."""
    N, args = _distill_args(logits, n_cols, teacher_ids, teacher_logits, temperature)
    _enqueue(lib().z2z_distill_grad, logits, *args, _dev(lse, torch.float32, N, "lse"), _dev(grad_loss, torch.float32, N, "grad_loss"),
             _like(grad, logits))


def z2z_set_distill_wait_limit(ns: int):
    """Nanoseconds after which a wait inside the distillation kernels gives up; 0 is the default, 400 ms."""
    _check(lib().z2z_set_distill_wait_limit(ns))


def z2z_xent_scratch_bytes(cfg: Config, N: int, grad_dtype: Optional[torch.dtype] = None):
    """(least, most) bytes of scratch for the cross entropy of N rows: of its losses alone, or with gradients of the tables
    in fp32 or bf16."""
    _need(grad_dtype in (None, torch.float32, torch.bfloat16), "grad_dtype must be fp32, bf16 or None")
    least, most = C.c_size_t(0), C.c_size_t(0)
    gd = -1 if grad_dtype is None else DTYPE_FP32 if grad_dtype == torch.float32 else DTYPE_BF16
    _check(lib().z2z_xent_scratch_bytes(C.byref(cfg), N, gd, C.byref(least), C.byref(most)))
    return least.value, most.value


def _xent_rows(cb: Codebook, hidden: torch.Tensor, row_seq, row_nvis, W_U, U_h, targets):
    c, dt, N = cb.cfg, _table_dtype(cb), hidden.shape[0]
    return N, (cb.handle, _dev(hidden, dt, N * c.d, "hidden"), N, _dev(row_seq, torch.int32, N, "row_seq"),
               _dev(row_nvis, torch.int32, N, "row_nvis"), _dev(W_U, dt, c.V * c.d, "W_U"), _cache(cb, U_h, dt, "U_h"),
               _dev(targets, torch.int32, N, "targets"))


def _xent_grads(cb: Codebook, N: int, accumulate: bool, grad_hidden, grad_WU, grad_Uh, scratch: torch.Tensor):
    c = cb.cfg
    some = grad_WU if grad_WU is not None else grad_Uh
    gt = torch.float32 if some is None else some.dtype
    _need(gt in (torch.float32, torch.bfloat16), "grad_WU and grad_Uh must be fp32 or bf16")
    # (without gradients of the tables their type is the session's: what its scratch is counted by)
    code = c.dtype if some is None else DTYPE_FP32 if gt == torch.float32 else DTYPE_BF16
    return (code, 1 if accumulate else 0, _dev(grad_hidden, _table_dtype(cb), N * c.d, "grad_hidden"), _dev(grad_WU, gt, c.V * c.d, "grad_WU"),
            _cache(cb, grad_Uh, gt, "grad_Uh"), _dev(scratch, torch.uint8, scratch.numel(), "scratch"), scratch.numel())


def z2z_xent_loss(cb: Codebook, hidden: torch.Tensor, row_seq: Optional[torch.Tensor], row_nvis: Optional[torch.Tensor], W_U: torch.Tensor,
                  U_h: Optional[torch.Tensor], targets: torch.Tensor, loss: torch.Tensor, lse: torch.Tensor, scratch: torch.Tensor):
    """Cross entropy of hidden [N, d] over the joint vocabulary against targets [N] -> loss [N], lse [N] (see z2z.h);
    scratch: uint8 tensor of z2z_xent_scratch_bytes."""
    N, args = _xent_rows(cb, hidden, row_seq, row_nvis, W_U, U_h, targets)
    _enqueue(lib().z2z_xent_loss, hidden, *args, _dev(loss, torch.float32, N, "loss"), _dev(lse, torch.float32, N, "lse"),
             _dev(scratch, torch.uint8, scratch.numel(), "scratch"), scratch.numel())


def z2z_xent_grad(cb: Codebook, hidden: torch.Tensor, row_seq: Optional[torch.Tensor], row_nvis: Optional[torch.Tensor], W_U: torch.Tensor,
                  U_h: Optional[torch.Tensor], targets: torch.Tensor, lse: torch.Tensor, grad_loss: Optional[torch.Tensor], accumulate: bool,
                  grad_hidden: Optional[torch.Tensor], grad_WU: Optional[torch.Tensor], grad_Uh: Optional[torch.Tensor], scratch: torch.Tensor):
    """Backward pass of z2z_xent_loss: lse as it left it, grad_loss [N] (None: ones) -> the gradients that are given."""
    N, args = _xent_rows(cb, hidden, row_seq, row_nvis, W_U, U_h, targets)
    _enqueue(lib().z2z_xent_grad, hidden, *args, _dev(lse, torch.float32, N, "lse"), _dev(grad_loss, torch.float32, N, "grad_loss"),
             *_xent_grads(cb, N, accumulate, grad_hidden, grad_WU, grad_Uh, scratch))


def z2z_xent_step(cb: Codebook, hidden: torch.Tensor, row_seq: Optional[torch.Tensor], row_nvis: Optional[torch.Tensor], W_U: torch.Tensor,
                  U_h: Optional[torch.Tensor], targets: torch.Tensor, row_weight: Optional[torch.Tensor], loss: torch.Tensor, lse: torch.Tensor,
                  accumulate: bool, grad_hidden: Optional[torch.Tensor], grad_WU: Optional[torch.Tensor], grad_Uh: Optional[torch.Tensor],
                  scratch: torch.Tensor):
    """Losses and the gradients of sum(row_weight * loss) in one call."""
    N, args = _xent_rows(cb, hidden, row_seq, row_nvis, W_U, U_h, targets)
    _enqueue(lib().z2z_xent_step, hidden, *args, _dev(row_weight, torch.float32, N, "row_weight"), _dev(loss, torch.float32, N, "loss"),
             _dev(lse, torch.float32, N, "lse"), *_xent_grads(cb, N, accumulate, grad_hidden, grad_WU, grad_Uh, scratch))


def z2z_set_xent_wait_limit(ns: int):
    """Nanoseconds after which a wait inside the cross entropy's kernels gives up; 0: the default."""
    _check(lib().z2z_set_xent_wait_limit(ns))


class GradTensors:
    """Records of gradient tensors for z2z_grad_clip, made once for tensors that stay where they are."""

    def __init__(self, records, tensors, device):
        self.records, self.device = records, device
        self._keep = tensors


def grad_tensors(grads: Sequence[torch.Tensor], outs: Optional[Sequence[Optional[torch.Tensor]]] = None) -> GradTensors:
    """Gradients (fp32 or bf16, contiguous, on one device) and where they go: outs[i] of the same size, fp32 or bf16, the
    gradient itself (in place), or None (counts for the norm alone); outs None: all in place."""
    grads = list(grads)
    outs = grads if outs is None else list(outs)
    _need(len(grads) == len(outs), "as many outputs as gradients are needed")
    codes = {torch.float32: DTYPE_FP32, torch.bfloat16: DTYPE_BF16}
    rec = (GradTensor * len(grads))()
    for r, g, o in zip(rec, grads, outs):
        for t in (g, o) if o is not None else (g,):
            _need(t.is_cuda and t.dtype in codes and t.is_contiguous() and t.numel() == g.numel() and t.device == grads[0].device,
                  "gradients and outputs must be contiguous device tensors of the same size, fp32 or bf16, on one device")
        r.d_grad, r.numel, r.grad_dtype = g.data_ptr(), g.numel(), codes[g.dtype]
        r.d_out, r.out_dtype = (o.data_ptr(), codes[o.dtype]) if o is not None else (None, r.grad_dtype)
    return GradTensors(rec, (grads, outs), grads[0].device if grads else None)


def z2z_grad_clip_scratch_bytes(tensors: GradTensors) -> int:
    out = C.c_size_t(0)
    _check(lib().z2z_grad_clip_scratch_bytes(len(tensors.records), C.byref(out)))
    return out.value


def z2z_grad_clip(tensors: GradTensors, scale: float, max_norm: float, norm: Optional[torch.Tensor], scratch: torch.Tensor):
    """norm [1] = |scale| * 2-norm of all gradients; outputs = scale * min(1, max_norm / (norm + 1e-6)) * gradient (see z2z.h);
    scratch: uint8 tensor of z2z_grad_clip_scratch_bytes."""
    _need(tensors.device is None or scratch.device == tensors.device, "scratch must be on the gradients' device")
    _enqueue(lib().z2z_grad_clip, scratch, tensors.records, len(tensors.records), scale, max_norm, _dev(norm, torch.float32, 1, "norm"),
             _dev(scratch, torch.uint8, scratch.numel(), "scratch"), scratch.numel())


def z2z_beam_select(cb: Codebook, beams: int, logits: torch.Tensor, lse: torch.Tensor, scores: torch.Tensor,
                    finished: Optional[torch.Tensor], eos: int, parent: torch.Tensor, code: torch.Tensor,
                    next_scores: torch.Tensor, next_finished: Optional[torch.Tensor] = None, active: Optional[torch.Tensor] = None):
    """Best continuations of every group of `beams` consecutive sequences, dealt to the group's slots (see z2z.h).
    logits [B, V + cap] and lse [B] as z2z_dynamic_logits stores them; finished / next_finished / active are uint8."""
    B = cb.cfg.B
    _enqueue(lib().z2z_beam_select, logits, cb.handle, beams, _dev(logits, torch.float32, B * (cb.cfg.V + cb.cfg.cap), "logits"),
             _dev(lse, torch.float32, B, "lse"), _dev(scores, torch.float32, B, "scores"), _dev(finished, torch.uint8, B, "finished"), eos,
             _dev(parent, torch.int32, B, "parent"), _dev(code, torch.int32, B, "code"), _dev(next_scores, torch.float32, B, "next_scores"),
             _dev(next_finished, torch.uint8, B, "next_finished"), _dev(active, torch.uint8, B, "active"))


def z2z_beam_reorder(cb: Codebook, parent: torch.Tensor, E_h: Optional[torch.Tensor], U_h: Optional[torch.Tensor],
                     E_h_f32: Optional[torch.Tensor] = None, U_h_f32: Optional[torch.Tensor] = None, states=()):
    """Sequence b takes over the codebook, caches and rows of sequence parent[b]; states: tensors [B, ...] of the caller's
    own whose row b belongs to sequence b."""
    c, dt = cb.cfg, _table_dtype(cb)
    rows = (SeqRows * len(states))() if states else None
    for r, t in zip(rows or (), states):
        _need(t.is_cuda and t.dim() > 0 and t.shape[0] == c.B and t[0].is_contiguous(), "a state must be a device tensor [B, ...] with contiguous rows")
        e = t.element_size()
        r.d_base, r.bytes = t.data_ptr(), t.numel() // c.B * e
        r.stride = t.stride(0) * e if c.B > 1 else r.bytes
    _enqueue(lib().z2z_beam_reorder, parent, cb.handle, _dev(parent, torch.int32, c.B, "parent"), _cache(cb, E_h, dt, "E_h"),
             _cache(cb, U_h, dt, "U_h"), _cache(cb, E_h_f32, torch.float32, "E_h_f32"), _cache(cb, U_h_f32, torch.float32, "U_h_f32"),
             rows, len(states))


def z2z_sample_filtered(logits: torch.Tensor, n_cols: torch.Tensor, top_k: int, top_p: float, temperature: float,
                        seed: int, step: int, choice: torch.Tensor, kept: Optional[torch.Tensor] = None,
                        row_base: int = 0):
    """logits [N, ld] fp32 (device), n_cols [N] int32 -> choice [N] int32 (and kept [N] int32)."""
    assert logits.dtype == torch.float32 and logits.dim() == 2
    _check(lib().z2z_sample_filtered(_ptr(logits), C.c_int32(logits.shape[0]), C.c_int64(logits.stride(0)),
                                     _ptr(n_cols), C.c_int32(top_k), C.c_float(top_p), C.c_float(temperature),
                                     C.c_uint64(seed), C.c_uint64(step), C.c_int32(row_base), _ptr(choice), _ptr(kept),
                                     _stream()))


def z2z_upload_rows(src_pinned: torch.Tensor, dst: torch.Tensor):
    """Pinned host tensor -> device tensor of the same size, by a kernel (see z2z.h)."""
    nbytes = src_pinned.numel() * src_pinned.element_size()
    assert src_pinned.is_pinned() and nbytes == dst.numel() * dst.element_size()
    _check(lib().z2z_upload_rows(_ptr(src_pinned), _ptr(dst), C.c_size_t(nbytes), _stream()))


def z2z_status(cb: Codebook):
    """(status bits [B], hypertoken counts [B]) as host int32 tensors; waits for the stream."""
    B = cb.cfg.B
    st = torch.empty(B, dtype=torch.int32)
    n = torch.empty(B, dtype=torch.int32)
    _check(lib().z2z_status(cb.handle, _ptr(st), _ptr(n), _stream()))
    return st, n


def z2z_codebook_read(cb: Codebook, b: int):
    """Codebook of sequence b on the host: (constituents [cap, M] int32, lengths [cap] int32)."""
    cons = torch.empty(cb.cfg.cap, cb.cfg.M, dtype=torch.int32)
    ln = torch.empty(cb.cfg.cap, dtype=torch.int32)
    _check(lib().z2z_codebook_read(cb.handle, C.c_int32(b), _ptr(cons), _ptr(ln), _stream()))
    return cons, ln


PROFILE_CLASSES = ["logits", "logits_merge", "lzw", "encoder_gemm", "encoder_other"]


def z2z_profile(cb: Codebook, enable: bool):
    _check(lib().z2z_profile(cb.handle, C.c_int32(1 if enable else 0)))


def z2z_profile_read(cb: Codebook):
    """({class: milliseconds}, {class: launches}) since the last read; waits for the stream."""
    n = len(PROFILE_CLASSES)
    ms = (C.c_double * n)()
    cnt = (C.c_int64 * n)()
    _check(lib().z2z_profile_read(cb.handle, C.c_int32(n), ms, cnt, _stream()))
    return ({k: ms[i] for i, k in enumerate(PROFILE_CLASSES)},
            {k: int(cnt[i]) for i, k in enumerate(PROFILE_CLASSES)})


def z2z_set_tensor_cores(cb: Codebook, enable):
    """0 / False: CUDA-core kernels; 1 / True: tensor-core kernels chosen by shape;
    2 + 16 * s: the CTA-pair logits kernel for every z2z_dynamic_logits call, with s column strips
    (0: chosen by shape)."""
    _check(lib().z2z_set_tensor_cores(cb.handle, C.c_int32(int(enable))))


def encoder_half_bytes(cfg: Config) -> int:
    """Bytes of scratch z2z_set_encoder_half_scratch needs for this configuration."""
    return 2 * cfg.enc_layers * (4 * cfg.d * cfg.d + 2 * cfg.d * cfg.enc_dff)


def z2z_set_encoder_half_scratch(cb: Codebook, scratch: Optional[torch.Tensor]):
    """Lend device memory (a uint8 tensor, 256-byte aligned) for fp16 copies of one encoder's
    linear-layer weights: long prompt-sized z2z_hyper_embed calls then run one tensor-core pass per
    k-step.  None returns to the two-part form.  The handle keeps a reference to the tensor."""
    cb._half_scratch = scratch
    nbytes = 0 if scratch is None else scratch.numel() * scratch.element_size()
    _check(lib().z2z_set_encoder_half_scratch(cb.handle, _ptr(scratch), C.c_size_t(nbytes)))


def z2z_logits_static_scratch(hidden: torch.Tensor, row_seq: Optional[torch.Tensor],
                              n_hyper: torch.Tensor, W_U: torch.Tensor,
                              U_h: Optional[torch.Tensor], cap: int,
                              lse: Optional[torch.Tensor], argmax: Optional[torch.Tensor],
                              max_logit: Optional[torch.Tensor]):
    """Joint logits + LSE / argmax / maximum without a session handle or workspace: for callers
    that cannot allocate device memory.  The partial reductions live in a fixed 2 MiB array
    inside the library (at most 1024 hidden rows per call).  ``n_hyper`` is a device int32 tensor
    [B] with the visible hypertokens of each sequence.  Calls that overlap on one GPU race on the
    shared array; the first call on a device should be made outside stream capture."""
    N, d = hidden.shape
    V = W_U.shape[0]
    B = n_hyper.shape[0]
    dt = DTYPE_FP32 if hidden.dtype == torch.float32 else DTYPE_BF16
    _check(lib().z2z_logits_static_scratch(_ptr(hidden), C.c_int32(N), _ptr(row_seq),
                                           _ptr(n_hyper), _ptr(W_U), _ptr(U_h), C.c_int32(V),
                                           C.c_int32(d), C.c_int32(B), C.c_int32(cap),
                                           C.c_int32(dt), _ptr(lse), _ptr(argmax),
                                           _ptr(max_logit), _stream()))
