"""The head's losses on torch tensors (include/vla_loss.h): cross entropy of tokens and distillation from a teacher's top
logits, each with its gradient.  Argument checks and output allocation only; all arithmetic is in the library's kernels.

Work goes to the current stream of the tensors' device.  `work` (uint8, from `loss_workspace`) is optional: without it a call
takes its workspace from torch's allocator, which keeps it for this call's stream.  Calls that may overlap, captured graphs that are
replayed side by side among them, need a workspace each.
"""
from __future__ import annotations

import ctypes as C
from functools import lru_cache
from typing import Optional

import torch

from . import binding as B

VLA_E_SHAPE, VLA_E_CONFIG = -3, -2
_DTYPES = {torch.float32: B.VLA_F32, torch.bfloat16: B.VLA_BF16}


def _refuse(code: int, msg: str):
    raise B.VlaError(code, msg)


def _rows(hidden, head, temperature: float) -> B.vla_head_rows:
    dtype = _DTYPES.get(hidden.dtype)
    if dtype is None or head.dtype != hidden.dtype:
        _refuse(VLA_E_CONFIG, f"hidden and head must both be float32 or bfloat16, not {hidden.dtype} and {head.dtype}")
    if hidden.dim() != 2 or head.dim() != 2 or hidden.shape[1] != head.shape[1]:
        _refuse(VLA_E_SHAPE, f"hidden [rows, d] and head [vocab, d], not {tuple(hidden.shape)} and {tuple(head.shape)}")
    if not hidden.is_cuda or head.device != hidden.device:
        _refuse(VLA_E_SHAPE, "hidden and head must be on one GPU")
    (T, d), V = hidden.shape, head.shape[0]
    (ld_h, one_h), (ld_w, one_w) = hidden.stride(), head.stride()
    if one_h != 1 or one_w != 1:
        _refuse(VLA_E_SHAPE, "the elements of a row of hidden and head must be next to each other")
    # (the stride of a single row means nothing)
    return B.vla_head_rows(hidden.data_ptr(), head.data_ptr(), ld_h if T > 1 else d, ld_w if V > 1 else d, T, d, V, dtype, temperature)


def _column(t, hidden, shape, dtype, name: str) -> int:
    if t.dtype != dtype or t.shape != shape or t.device != hidden.device or not t.is_contiguous():
        _refuse(VLA_E_SHAPE, f"{name} must be a contiguous {dtype} tensor {tuple(shape)} on {hidden.device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _labels(hidden, labels):
    return (_column(labels, hidden, hidden.shape[:1], torch.int32, "labels"),), 0


def _teacher(hidden, top_logits, top_ids):
    if top_ids.dim() != 2:
        _refuse(VLA_E_SHAPE, f"top_ids must be [rows, n], not {tuple(top_ids.shape)}")
    shape = torch.Size((hidden.shape[0], top_ids.shape[1]))
    return (_column(top_logits, hidden, shape, torch.float32, "top_logits"), _column(top_ids, hidden, shape, torch.int32, "top_ids"),
            shape[1]), shape[1]


@lru_cache(maxsize=4096)
def _workspace(T: int, d: int, V: int, dtype: int, n_top: int, grad: bool) -> int:
    return B.vla_loss_workspace(B.vla_head_rows(0, 0, 0, 0, T, d, V, dtype, 0.0), n_top, grad)


def loss_workspace(hidden, head, n_top: int = 0, grad: bool = False) -> int:
    """Bytes of `work` for such tensors: n_top 0 for the token losses, grad for the gradient's call."""
    r = _rows(hidden, head, 0.0)
    return _workspace(r.n_rows, r.d_model, r.vocab, r.dtype, n_top, bool(grad))


def _call(name: str, rows, targets, n_top: int, grad: bool, hidden, work, args):
    device = hidden.device
    if work is None:
        work = torch.empty(_workspace(rows.n_rows, rows.d_model, rows.vocab, rows.dtype, n_top, grad), dtype=torch.uint8, device=device)
    elif work.dtype != torch.uint8 or work.device != device or not work.is_contiguous():
        _refuse(VLA_E_SHAPE, f"work must be a contiguous uint8 tensor on {device}")
    call = getattr(B.lib(), name)
    a = (C.byref(rows), *targets, *args, work.data_ptr(), work.numel())
    if device.index == torch.cuda.current_device():
        rc = call(*a, torch._C._cuda_getCurrentRawStream(device.index))   # (torch.cuda.current_stream without its wrapper object)
    else:
        with torch.cuda.device(device):
            rc = call(*a, torch._C._cuda_getCurrentRawStream(device.index))
    if rc:
        raise B.VlaError(rc, name)


def _loss(name, hidden, head, targets, n_top, temperature, work):
    rows = _rows(hidden, head, temperature)
    loss, lse = torch.empty((2, rows.n_rows), dtype=torch.float32, device=hidden.device).unbind(0)
    _call(name, rows, targets, n_top, False, hidden, work, (loss.data_ptr(), lse.data_ptr()))
    return loss, lse


def _grad(name, hidden, head, targets, n_top, lse, grad_loss, temperature, want_hidden, want_head, work):
    rows = _rows(hidden, head, temperature)
    shape = hidden.shape[:1]
    columns = _column(lse, hidden, shape, torch.float32, "lse"), _column(grad_loss, hidden, shape, torch.float32, "grad_loss")
    gh = torch.empty(hidden.shape, dtype=hidden.dtype, device=hidden.device) if want_hidden else None
    gw = torch.empty(head.shape, dtype=head.dtype, device=head.device) if want_head else None
    _call(name, rows, targets, n_top, True, hidden, work, (*columns, gh.data_ptr() if want_hidden else None,
                                                           gw.data_ptr() if want_head else None))
    return gh, gw


def token_loss(hidden, head, labels, temperature: float = 0.0, work: Optional[torch.Tensor] = None):
    """(loss, lse) [rows] float32 of labels [rows] int32: lse - z[label], z = hidden head^T / temperature (0 means 1, others lie
    between 2^-40 and 2^40).  A label outside [0, vocab): no target, 0."""
    return _loss("vla_token_loss", hidden, head, *_labels(hidden, labels), temperature, work)


def token_loss_grad(hidden, head, labels, lse, grad_loss, temperature: float = 0.0, want_hidden: bool = True,
                    want_head: bool = True, work: Optional[torch.Tensor] = None):
    """(grad_hidden, grad_head) of sum grad_loss * loss; lse as token_loss returned it.  None for what is not wanted."""
    return _grad("vla_token_loss_grad", hidden, head, *_labels(hidden, labels), lse, grad_loss, temperature, want_hidden, want_head,
                 work)


def distill_loss(hidden, head, top_logits, top_ids, temperature: float = 0.0, work: Optional[torch.Tensor] = None):
    """(loss, lse) [rows] float32: KL(p || softmax z), p a softmax of a row's teacher logits [rows, n] / temperature at
    ids [rows, n] int32.  Entries with an id outside [0, vocab) or a logit of -inf are not there, equal ids add up."""
    return _loss("vla_distill_loss", hidden, head, *_teacher(hidden, top_logits, top_ids), temperature, work)


def distill_loss_grad(hidden, head, top_logits, top_ids, lse, grad_loss, temperature: float = 0.0, want_hidden: bool = True,
                      want_head: bool = True, work: Optional[torch.Tensor] = None):
    """(grad_hidden, grad_head) of sum grad_loss * loss; lse as distill_loss returned it.  None for what is not wanted."""
    return _grad("vla_distill_loss_grad", hidden, head, *_teacher(hidden, top_logits, top_ids), lse, grad_loss, temperature,
                 want_hidden, want_head, work)
