"""What stands around the MoE layer in a decoder block: calls on torch tensors.

``dispatch`` / ``combine`` (tokens sorted by expert and back, routing weights applied) and their gradients, ``norm_join``
(norm behind a block, gate, residual scale, norm in front of the next) and its gradient, ``quantize_linear`` / ``linear``
(products with a 4-bit matrix that has group scales).  ``include/dynamo.h`` has the definitions; argument checks, result tensors and
the stream are ``csrc/torch_binding.cpp``'s.

Tensors are contiguous, on one CUDA device, 16-byte aligned; they may be on another device than the current one.  Work goes to
the current stream of the tensors' device, and a tensor that another stream wrote or will free is the caller's to order, as with
torch's own functions.  A wrong tensor raises ``ValueError`` before anything is launched, what the library refuses
``binding.DynamoError``.  The functions do not take part in automatic differentiation: gradients are calls of their own, and a tensor
that requires its gradient is refused (``ValueError``) unless torch records none (``torch.no_grad()``, ``detach()``).
Results and scratch memory come from torch's allocator, so a call may be captured in a graph.  A tensor that is given for a result (out,
d_rows, r_out, n_out) overlaps no input and no other result, but r_out may be r.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

import torch

from .binding import BF16, F32, OK, STATUS_NAMES, DynamoError, load

_native = None
_ERR_TIMEOUT = STATUS_NAMES.index("ERR_TIMEOUT")


def _lib():
    """The compiled calls; raises if they have not been built (no other path exists)."""
    global _native
    if _native is None:
        load()
        from . import _native as mod   # beside the library, which it calls

        mod.set_error(DynamoError)
        _native = mod
    return _native


class Dispatched(NamedTuple):
    """rows [T k, d] (None without x), offsets int32 [E + 1], perm int32 [T k], pos int32 [T, k]."""
    rows: Optional[torch.Tensor]
    offsets: torch.Tensor
    perm: torch.Tensor
    pos: torch.Tensor


# ---- tokens sorted by expert and back ------------------------------------------------------------------------------------

def dispatch(topk_idx: torch.Tensor, n_experts: int, x: Optional[torch.Tensor] = None,
             out: Optional[Tuple] = None) -> Dispatched:
    """Sort of the (token, slot) pairs of topk_idx int32 [T, k] by expert; with x [T, d] also the tokens' rows in that order.
    Indices outside [0, n_experts) drop their pair.  Rows and entries of perm behind the last kept pair are not written.
    out: buffers like the result's (a tuple of the four) to use instead of new ones."""
    return Dispatched._make(_lib().dispatch(topk_idx, n_experts, x, out))


def combine(rows: torch.Tensor, pos: torch.Tensor, topk_w: Optional[torch.Tensor] = None, y_dtype: Optional[int] = None,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y[t] = sum_j topk_w[t, j] * rows[pos[t, j]] ([T, d]; ones without topk_w).  y_dtype: BF16 or F32, rows' type by default."""
    return _lib().combine(rows, pos, topk_w, y_dtype, out)


def dispatch_backward(d_rows: torch.Tensor, pos: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of dispatch's x [T, d] from that of its rows."""
    return _lib().combine(d_rows, pos, None, None, out)


def combine_backward(dy: torch.Tensor, rows: torch.Tensor, pos: torch.Tensor, topk_w: Optional[torch.Tensor] = None,
                     d_rows: Optional[torch.Tensor] = None, want_d_w: bool = True):
    """Gradients (d_rows [T k, d], d_w fp32 [T, k] or None) of combine.  Rows that no pair names are not written."""
    return _lib().combine_backward(dy, rows, pos, topk_w, d_rows, want_d_w)


# ---- a block's output joined with the residual stream --------------------------------------------------------------------

def norm_join(r: torch.Tensor, y: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
              gate: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None, post_norm: bool = True,
              pre_norm: bool = True, res_scale: float = 1.0, block_scale: float = 1.0, eps: float = 1e-6, n_dtype: int = BF16,
              want_stats: bool = False, r_out: Optional[torch.Tensor] = None, n_out: Optional[torch.Tensor] = None):
    """(r_out, n[, stats]): r_out = res_scale * r + block_scale * gate * norm(y) * w_post, n = norm(r_out) * w_pre, [T, d] each.

    gate: [d] or fp32 [T, 1].  Without y, r_out is r itself; without post_norm y is taken as it is; without pre_norm n is None.
    want_stats: also the row factors fp32 [T, 2] for the gradient.  r_out may be r (the stream updated in place)."""
    return _lib().norm_join(r, y, w_post, gate, w_pre, post_norm, pre_norm, res_scale, block_scale, eps, n_dtype, want_stats,
                            r_out, n_out)


def norm_join_backward(d_n: Optional[torch.Tensor], d_r_out: Optional[torch.Tensor], r: torch.Tensor, y: Optional[torch.Tensor],
                       stats: torch.Tensor, w_post: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                       w_pre: Optional[torch.Tensor] = None, post_norm: bool = True, pre_norm: bool = True,
                       res_scale: float = 1.0, block_scale: float = 1.0, eps: float = 1e-6) -> dict:
    """Gradients of norm_join from those of n (None without pre_norm) and of r_out (None: zero), with what the forward had and
    the stats it gave.  dict(d_r, d_y, d_w_post, d_gate, d_w_pre), None for what is not there; those of weights and gate in fp32."""
    d_r, d_y, d_w_post, d_gate, d_w_pre = _lib().norm_join_backward(d_n, d_r_out, stats, r, y, w_post, gate, w_pre, post_norm,
                                                                    pre_norm, res_scale, block_scale, eps)
    return {"d_r": d_r, "d_y": d_y, "d_w_post": d_w_post, "d_gate": d_gate, "d_w_pre": d_w_pre}


# ---- products with a 4-bit matrix ----------------------------------------------------------------------------------------

def quantize_linear(w: torch.Tensor, group_size: int = 128) -> Tuple[torch.Tensor, torch.Tensor]:
    """(codes uint8 [N, K / 2], params fp16 [N, K / group_size, 2]) of w bf16 [N, K]: the experts' quantizer at 4 bits."""
    return _lib().quantize_linear(w, group_size)


def linear(x: torch.Tensor, codes: torch.Tensor, params: torch.Tensor, y_dtype: int = F32,
           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [T, N] = x bf16 [T, K] times the transposed matrix that codes and params stand for."""
    return _lib().linear(x, codes, params, y_dtype, out)


def poll_linear_status(device=None) -> int:
    """Waits for the device's (the current one's) current stream.  0, or the library's ERR_TIMEOUT if a bounded wait of ``linear`` has
    expired on it: results that are NaN are lost.  Every caller is told, until ``clear_linear_status``.  Raises DynamoError if the
    status cannot be read."""
    with torch.cuda.device(device):
        st = load().dynamo_linear_poll_status(torch.cuda.current_stream().cuda_stream)
    if st not in (OK, _ERR_TIMEOUT):
        raise DynamoError(st, "dynamo_linear_poll_status")
    return st


def clear_linear_status(device=None) -> None:
    """Waits for the device's current stream and sets the status of ``poll_linear_status`` back to 0, for all users of the device."""
    with torch.cuda.device(device):
        st = load().dynamo_linear_clear_status(torch.cuda.current_stream().cuda_stream)
    if st != OK:
        raise DynamoError(st, "dynamo_linear_clear_status")
