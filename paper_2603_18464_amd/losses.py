"""The head's losses on torch tensors (include/vla_loss.h): cross entropy of tokens and distillation from a teacher's top
logits, each with its gradient.  Argument checks and output allocation only; all arithmetic is in the library's kernels.

Work goes to the current stream of the tensors' device.  `work` (uint8, from `loss_workspace`) is optional: without it a call
takes its workspace from torch's allocator, which keeps it for this call's stream.  Calls that may overlap, captured graphs that are
replayed side by side among them, need a workspace each.
"""
from __future__ import annotations

from typing import Optional

from . import binding as B

VLA_E_SHAPE, VLA_E_CONFIG = -3, -2


def _refuse(code: int, msg: str):
    raise B.VlaError(code, msg)


def _rows(hidden, head, temperature: float) -> B.vla_head_rows:
    import torch
    if hidden.dtype not in (torch.float32, torch.bfloat16) or head.dtype != hidden.dtype:
        _refuse(VLA_E_CONFIG, f"hidden and head must both be float32 or bfloat16, not {hidden.dtype} and {head.dtype}")
    if hidden.dim() != 2 or head.dim() != 2 or hidden.shape[1] != head.shape[1]:
        _refuse(VLA_E_SHAPE, f"hidden [rows, d] and head [vocab, d], not {tuple(hidden.shape)} and {tuple(head.shape)}")
    if not hidden.is_cuda or head.device != hidden.device:
        _refuse(VLA_E_SHAPE, "hidden and head must be on one GPU")
    d = hidden.shape[1]
    for name, t in (("hidden", hidden), ("head", head)):
        if t.numel() and t.stride(1) != 1:
            _refuse(VLA_E_SHAPE, f"the elements of a row of {name} must be next to each other")
    # (the stride of a single row means nothing)
    ld = [t.stride(0) if t.shape[0] > 1 else d for t in (hidden, head)]
    return B.vla_head_rows(hidden.data_ptr(), head.data_ptr(), ld[0], ld[1], hidden.shape[0], d, head.shape[0],
                           B.VLA_F32 if hidden.dtype == torch.float32 else B.VLA_BF16, float(temperature))


def _column(t, like, shape, dtype, name: str):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or t.device != like.device or not t.is_contiguous():
        _refuse(VLA_E_SHAPE, f"{name} must be a contiguous {dtype} tensor {tuple(shape)} on {like.device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def _targets(hidden, labels=None, top_logits=None, top_ids=None):
    import torch
    if labels is not None:
        return (_column(labels, hidden, hidden.shape[:1], torch.int32, "labels"),)
    if top_ids.dim() != 2:
        _refuse(VLA_E_SHAPE, f"top_ids must be [rows, n], not {tuple(top_ids.shape)}")
    shape = (hidden.shape[0], top_ids.shape[1])
    return (_column(top_logits, hidden, shape, torch.float32, "top_logits"), _column(top_ids, hidden, shape, torch.int32, "top_ids"),
            shape[1])


def _work(rows, n_top: int, grad: bool, hidden, work):
    import torch
    need = B.vla_loss_workspace(rows, n_top, grad)
    if work is None:
        return torch.empty(need, dtype=torch.uint8, device=hidden.device)
    if work.dtype != torch.uint8 or work.device != hidden.device or not work.is_contiguous():
        _refuse(VLA_E_SHAPE, f"work must be a contiguous uint8 tensor on {hidden.device}")
    return work


def loss_workspace(hidden, head, n_top: int = 0, grad: bool = False) -> int:
    """Bytes of `work` for such tensors: n_top 0 for the token losses, grad for the gradient's call."""
    return B.vla_loss_workspace(_rows(hidden, head, 0.0), n_top, grad)


def _loss(call, hidden, head, targets, temperature, work):
    import torch
    rows = _rows(hidden, head, temperature)
    with torch.cuda.device(hidden.device):
        work = _work(rows, targets[2] if len(targets) == 3 else 0, False, hidden, work)
        out = torch.empty((2, hidden.shape[0]), dtype=torch.float32, device=hidden.device)
        call(rows, *targets, out[0], out[1], work, torch.cuda.current_stream().cuda_stream)
    return out[0], out[1]


def _grad(call, hidden, head, targets, lse, grad_loss, temperature, want_hidden, want_head, work):
    import torch
    rows = _rows(hidden, head, temperature)
    _column(lse, hidden, hidden.shape[:1], torch.float32, "lse")
    _column(grad_loss, hidden, hidden.shape[:1], torch.float32, "grad_loss")
    with torch.cuda.device(hidden.device):
        work = _work(rows, targets[2] if len(targets) == 3 else 0, True, hidden, work)
        gh = torch.empty(hidden.shape, dtype=hidden.dtype, device=hidden.device) if want_hidden else None
        gw = torch.empty(head.shape, dtype=head.dtype, device=head.device) if want_head else None
        call(rows, *targets, lse, grad_loss, gh, gw, work, torch.cuda.current_stream().cuda_stream)
    return gh, gw


def token_loss(hidden, head, labels, temperature: float = 0.0, work: Optional["object"] = None):
    """(loss, lse) [rows] float32 of labels [rows] int32: lse - z[label], z = hidden head^T / temperature (0 means 1).
    A label outside [0, vocab): no target, 0."""
    return _loss(B.vla_token_loss, hidden, head, _targets(hidden, labels=labels), temperature, work)


def token_loss_grad(hidden, head, labels, lse, grad_loss, temperature: float = 0.0, want_hidden: bool = True,
                    want_head: bool = True, work: Optional["object"] = None):
    """(grad_hidden, grad_head) of sum grad_loss * loss; lse as token_loss returned it.  None for what is not wanted."""
    return _grad(B.vla_token_loss_grad, hidden, head, _targets(hidden, labels=labels), lse, grad_loss, temperature,
                 want_hidden, want_head, work)


def distill_loss(hidden, head, top_logits, top_ids, temperature: float = 0.0, work: Optional["object"] = None):
    """(loss, lse) [rows] float32: KL(p || softmax z), p a softmax of a row's teacher logits [rows, n] / temperature at
    ids [rows, n] int32.  Entries with an id outside [0, vocab) or a logit of -inf are not there, equal ids add up."""
    return _loss(B.vla_distill_loss, hidden, head, _targets(hidden, top_logits=top_logits, top_ids=top_ids), temperature, work)


def distill_loss_grad(hidden, head, top_logits, top_ids, lse, grad_loss, temperature: float = 0.0, want_hidden: bool = True,
                      want_head: bool = True, work: Optional["object"] = None):
    """(grad_hidden, grad_head) of sum grad_loss * loss; lse as distill_loss returned it.  None for what is not wanted."""
    return _grad(B.vla_distill_loss_grad, hidden, head, _targets(hidden, top_logits=top_logits, top_ids=top_ids), lse, grad_loss,
                 temperature, want_hidden, want_head, work)
