"""What stands around the MoE layer in a decoder block: calls on torch tensors (argument checks and marshalling only).

``dispatch`` / ``combine`` (tokens sorted by expert and back, routing weights applied) and their gradients, ``norm_join``
(norm behind a block, gate, residual scale, norm in front of the next) and its gradient, ``quantize_linear`` / ``linear``
(products with a 4-bit matrix that has group scales).  ``include/dynamo.h`` has the definitions.

Tensors are contiguous, on one CUDA device, 16-byte aligned; they may be on another device than the current one.  Work goes to
the current stream of the tensors' device, and a tensor that another stream wrote or will free is the caller's to order, as with
torch's own functions.  A wrong tensor raises ``ValueError`` before anything is launched, what the library refuses
``binding.DynamoError``.  The functions do not take part in automatic differentiation: gradients are calls of their own.
Results and scratch memory come from torch's allocator, so a call may be captured in a graph.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Tuple

import torch

from .binding import (BF16, F32, GATE_CHANNEL, GATE_NONE, GATE_TOKEN, OK, DynamoError, JoinDesc, load)

# The handle alone: torch.cuda.current_stream() makes an object around it, 3.2 of the 14 us that a small call took on the host.
_raw_stream = torch._C._cuda_getCurrentRawStream

_CODE = {torch.bfloat16: BF16, torch.float32: F32}
_TYPE = {BF16: torch.bfloat16, F32: torch.float32}


class Dispatched(NamedTuple):
    """rows [T k, d] (None without x), offsets int32 [E + 1], perm int32 [T k], pos int32 [T, k]."""
    rows: Optional[torch.Tensor]
    offsets: torch.Tensor
    perm: torch.Tensor
    pos: torch.Tensor


def _want(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _tensor(t: torch.Tensor, name: str, device, dtype=None, shape=None) -> None:
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: a tensor is wanted")
    if t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous tensor on {device} is wanted")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: {dtype} is wanted")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(shape)} is wanted")


def _device(t: torch.Tensor, name: str):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor is wanted")
    return t.device


def _real(t: torch.Tensor, name: str) -> int:
    code = _CODE.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: bfloat16 or float32 is wanted")
    return code


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _call(name: str, device, *args) -> None:
    """The library's call on the current stream of `device`."""
    fn, index = getattr(load(), name), device.index
    if index == torch.cuda.current_device():
        st = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            st = fn(*args, _raw_stream(index))
    if st != OK:
        raise DynamoError(st, name)


# ---- tokens sorted by expert and back ------------------------------------------------------------------------------------

def dispatch(topk_idx: torch.Tensor, n_experts: int, x: Optional[torch.Tensor] = None,
             out: Optional[Tuple] = None) -> Dispatched:
    """Sort of the (token, slot) pairs of topk_idx int32 [T, k] by expert; with x [T, d] also the tokens' rows in that order.
    Indices outside [0, n_experts) drop their pair.  Rows and entries of perm behind the last kept pair are not written.
    out: buffers like the result's to use instead of new ones."""
    device = _device(topk_idx, "topk_idx")
    _tensor(topk_idx, "topk_idx", device, torch.int32)
    _want(topk_idx.dim() == 2, "topk_idx: [T, k] is wanted")
    T, k = topk_idx.shape
    d = code = 0
    if x is not None:
        _tensor(x, "x", device)
        _want(x.dim() == 2 and x.shape[0] == T, "x: [T, d] is wanted")
        d, code = x.shape[1], _real(x, "x")
    if out is None:
        rows = None if x is None else torch.empty((T * k, d), dtype=x.dtype, device=device)
        offsets = torch.empty((n_experts + 1,), dtype=torch.int32, device=device)
        perm = torch.empty((T * k,), dtype=torch.int32, device=device)
        pos = torch.empty((T, k), dtype=torch.int32, device=device)
    else:
        rows, offsets, perm, pos = out
        _want((rows is None) == (x is None), "out.rows: given with x alone")
        if x is not None:
            _tensor(rows, "out.rows", device, x.dtype, (T * k, d))
        _tensor(offsets, "out.offsets", device, torch.int32, (n_experts + 1,))
        _tensor(perm, "out.perm", device, torch.int32, (T * k,))
        _tensor(pos, "out.pos", device, torch.int32, (T, k))
    need = ctypes.c_size_t(0)
    st = load().dynamo_dispatch_workspace_bytes(T, n_experts, k, ctypes.byref(need))
    if st != OK:
        raise DynamoError(st, "dynamo_dispatch_workspace_bytes")
    ws = torch.empty((need.value,), dtype=torch.uint8, device=device) if need.value else None
    _call("dynamo_dispatch", device, topk_idx.data_ptr(), T, n_experts, k, _ptr(x), d, code, offsets.data_ptr(),
          perm.data_ptr(), pos.data_ptr(), _ptr(rows), _ptr(ws), need.value)
    return Dispatched(rows, offsets, perm, pos)


def combine(rows: torch.Tensor, pos: torch.Tensor, topk_w: Optional[torch.Tensor] = None, y_dtype: Optional[int] = None,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y[t] = sum_j topk_w[t, j] * rows[pos[t, j]] ([T, d]; ones without topk_w).  y_dtype: BF16 or F32, rows' type by default."""
    device = _device(rows, "rows")
    _tensor(rows, "rows", device)
    _tensor(pos, "pos", device, torch.int32)
    _want(rows.dim() == 2 and pos.dim() == 2, "rows: [T k, d] and pos: [T, k] are wanted")
    T, k = pos.shape
    d = rows.shape[1]
    _want(rows.shape[0] == T * k, "rows: [T k, d] is wanted")
    code = _real(rows, "rows")
    if topk_w is not None:
        _tensor(topk_w, "topk_w", device, torch.float32, (T, k))
    y_code = code if y_dtype is None else y_dtype
    _want(y_code in _TYPE, "y_dtype: BF16 or F32 is wanted")
    if out is None:
        out = rows.new_empty((T, d)) if y_code == code else torch.empty((T, d), dtype=_TYPE[y_code], device=device)
    else:
        _tensor(out, "out", device, _TYPE[y_code], (T, d))
    _call("dynamo_combine", device, rows.data_ptr(), code, pos.data_ptr(), _ptr(topk_w), T, k, d, out.data_ptr(), y_code)
    return out


def dispatch_backward(d_rows: torch.Tensor, pos: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of dispatch's x [T, d] from that of its rows."""
    return combine(d_rows, pos, out=out)


def combine_backward(dy: torch.Tensor, rows: torch.Tensor, pos: torch.Tensor, topk_w: Optional[torch.Tensor] = None,
                     d_rows: Optional[torch.Tensor] = None, want_d_w: bool = True):
    """Gradients (d_rows [T k, d], d_w fp32 [T, k] or None) of combine.  Rows that no pair names are not written."""
    device = _device(rows, "rows")
    _tensor(rows, "rows", device)
    _tensor(pos, "pos", device, torch.int32)
    _want(rows.dim() == 2 and pos.dim() == 2, "rows: [T k, d] and pos: [T, k] are wanted")
    T, k = pos.shape
    d = rows.shape[1]
    _want(rows.shape[0] == T * k, "rows: [T k, d] is wanted")
    _tensor(dy, "dy", device, None, (T, d))
    dy_code, code = _real(dy, "dy"), _real(rows, "rows")
    if topk_w is not None:
        _tensor(topk_w, "topk_w", device, torch.float32, (T, k))
    if d_rows is None:
        d_rows = torch.empty_like(rows)
    else:
        _tensor(d_rows, "d_rows", device, rows.dtype, rows.shape)
    d_w = None if not want_d_w else torch.empty((T, k), dtype=torch.float32, device=device) if topk_w is None else torch.empty_like(topk_w)
    _call("dynamo_combine_backward", device, dy.data_ptr(), dy_code, rows.data_ptr(), code, pos.data_ptr(), _ptr(topk_w), T, k,
          d, d_rows.data_ptr(), _ptr(d_w))
    return d_rows, d_w


# ---- a block's output joined with the residual stream --------------------------------------------------------------------

def _join_desc(r, y, w_post, gate, w_pre, post_norm, pre_norm, res_scale, block_scale, eps, n_code) -> JoinDesc:
    device = _device(r, "r")
    _tensor(r, "r", device)
    _want(r.dim() == 2, "r: [T, d] is wanted")
    T, d = r.shape
    _want(y is not None or (gate is None and w_post is None), "gate and w_post go with y")
    _want(post_norm or w_post is None, "w_post goes with post_norm")
    _want(pre_norm or w_pre is None, "w_pre goes with pre_norm")
    _want(n_code in _TYPE, "n_dtype: BF16 or F32 is wanted")
    y_code = r_code = _real(r, "r")
    if y is not None:
        _tensor(y, "y", device, None, (T, d))
        y_code = _real(y, "y")
    kind, w_type = GATE_NONE, None
    if gate is not None:
        _want(isinstance(gate, torch.Tensor) and gate.dim() in (1, 2), "gate: [d] or [T, 1] is wanted")
        if gate.dim() == 2:
            kind = GATE_TOKEN
            _tensor(gate, "gate", device, torch.float32, (T, 1))
        else:
            kind, w_type = GATE_CHANNEL, gate.dtype
            _tensor(gate, "gate", device, None, (d,))
    for name, w in (("w_post", w_post), ("w_pre", w_pre)):
        if w is not None:
            w_type = w.dtype if w_type is None else w_type
            _tensor(w, name, device, w_type, (d,))
    w_code = F32 if w_type is None else _CODE.get(w_type)
    _want(w_code is not None, "weights: bfloat16 or float32 is wanted")
    return JoinDesc(d, y_code, r_code, n_code, w_code, kind, 1 if post_norm and y is not None else 0, 1 if pre_norm else 0, res_scale,
                    block_scale, eps)


def norm_join(r: torch.Tensor, y: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
              gate: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None, post_norm: bool = True,
              pre_norm: bool = True, res_scale: float = 1.0, block_scale: float = 1.0, eps: float = 1e-6, n_dtype: int = BF16,
              want_stats: bool = False, r_out: Optional[torch.Tensor] = None, n_out: Optional[torch.Tensor] = None):
    """(r_out, n[, stats]): r_out = res_scale * r + block_scale * gate * norm(y) * w_post, n = norm(r_out) * w_pre, [T, d] each.

    gate: [d] or [T, 1].  Without y, r_out is r itself; without post_norm y is taken as it is; without pre_norm n is None.
    want_stats: also the row factors fp32 [T, 2] for the gradient.  r_out may be r (the stream updated in place)."""
    desc = _join_desc(r, y, w_post, gate, w_pre, post_norm, pre_norm, res_scale, block_scale, eps, n_dtype)
    device, shape = r.device, r.shape
    if y is None:
        _want(r_out is None, "r_out goes with y")
    elif r_out is None:
        r_out = torch.empty_like(r)
    else:
        _tensor(r_out, "r_out", device, r.dtype, shape)
    if not pre_norm:
        _want(n_out is None, "n_out goes with pre_norm")
    elif n_out is None:
        n_out = r.new_empty(shape) if n_dtype == desc.r_dtype else torch.empty(shape, dtype=_TYPE[n_dtype], device=device)
    else:
        _tensor(n_out, "n_out", device, _TYPE[n_dtype], shape)
    stats = torch.empty((shape[0], 2), dtype=torch.float32, device=device) if want_stats else None
    _call("dynamo_norm_join_forward", device, ctypes.byref(desc), r.data_ptr(), _ptr(y), _ptr(w_post), _ptr(gate), _ptr(w_pre),
          shape[0], _ptr(r_out), _ptr(n_out), _ptr(stats))
    res = (r if y is None else r_out, n_out)
    return res + (stats,) if want_stats else res


def norm_join_backward(d_n: Optional[torch.Tensor], d_r_out: Optional[torch.Tensor], r: torch.Tensor, y: Optional[torch.Tensor],
                       stats: torch.Tensor, w_post: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                       w_pre: Optional[torch.Tensor] = None, post_norm: bool = True, pre_norm: bool = True,
                       res_scale: float = 1.0, block_scale: float = 1.0, eps: float = 1e-6) -> dict:
    """Gradients of norm_join from those of n (None without pre_norm) and of r_out (None: zero), with what the forward had and
    the stats it gave.  dict(d_r, d_y, d_w_post, d_gate, d_w_pre), None for what is not there; those of weights and gate in fp32."""
    _want((d_n is not None) == bool(pre_norm), "d_n goes with pre_norm")
    _want(d_n is not None or d_r_out is not None, "d_r_out: wanted without pre_norm")
    n_code = BF16 if d_n is None else _CODE.get(getattr(d_n, "dtype", None), -1)
    desc = _join_desc(r, y, w_post, gate, w_pre, post_norm, pre_norm, res_scale, block_scale, eps, n_code)
    device, (T, d) = r.device, r.shape
    if d_n is not None:
        _tensor(d_n, "d_n", device, None, (T, d))
    if d_r_out is not None:
        _tensor(d_r_out, "d_r_out", device, r.dtype, (T, d))
    _tensor(stats, "stats", device, torch.float32, (T, 2))

    def sums(like):
        return None if like is None else stats.new_empty(like.shape)

    d_r = torch.empty_like(r)
    d_y = None if y is None else torch.empty_like(y)
    d_w_post, d_gate, d_w_pre = sums(w_post), sums(gate), sums(w_pre)
    ws, need = None, ctypes.c_size_t(0)
    if d_w_post is not None or d_w_pre is not None or (d_gate is not None and gate.dim() == 1):
        st = load().dynamo_norm_join_workspace_bytes(ctypes.byref(desc), T, ctypes.byref(need))
        if st != OK:
            raise DynamoError(st, "dynamo_norm_join_workspace_bytes")
        ws = torch.empty((need.value,), dtype=torch.uint8, device=device)
    _call("dynamo_norm_join_backward", device, ctypes.byref(desc), _ptr(d_n), _ptr(d_r_out), r.data_ptr(), _ptr(y), stats.data_ptr(),
          _ptr(w_post), _ptr(gate), _ptr(w_pre), T, d_r.data_ptr(), _ptr(d_y), _ptr(d_w_post), _ptr(d_gate), _ptr(d_w_pre),
          _ptr(ws), need.value)
    return {"d_r": d_r, "d_y": d_y, "d_w_post": d_w_post, "d_gate": d_gate, "d_w_pre": d_w_pre}


# ---- products with a 4-bit matrix ----------------------------------------------------------------------------------------

def quantize_linear(w: torch.Tensor, group_size: int = 128) -> Tuple[torch.Tensor, torch.Tensor]:
    """(codes uint8 [N, K / 2], params fp16 [N, K / group_size, 2]) of w bf16 [N, K]: the experts' quantizer at 4 bits."""
    device = _device(w, "w")
    _tensor(w, "w", device, torch.bfloat16)
    _want(w.dim() == 2, "w: [N, K] is wanted")
    _want(group_size in (64, 128) and w.shape[1] % group_size == 0, "group_size: 64 or 128, a divisor of K, is wanted")
    N, K = w.shape
    codes = torch.empty((N, K // 2), dtype=torch.uint8, device=device)
    params = torch.empty((N, K // group_size, 2), dtype=torch.float16, device=device)
    _call("dynamo_linear_quantize", device, w.data_ptr(), N, K, group_size, codes.data_ptr(), params.data_ptr())
    return codes, params


def linear(x: torch.Tensor, codes: torch.Tensor, params: torch.Tensor, y_dtype: int = F32,
           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [T, N] = x bf16 [T, K] times the transposed matrix that codes and params stand for."""
    device = _device(x, "x")
    _tensor(x, "x", device, torch.bfloat16)
    _want(x.dim() == 2, "x: [T, K] is wanted")
    T, K = x.shape
    _tensor(params, "params", device, torch.float16)
    _want(params.dim() == 3 and params.shape[2] == 2, "params: [N, K / group_size, 2] is wanted")
    N, groups = params.shape[0], params.shape[1]
    _want(groups > 0 and K % groups == 0, "params: [N, K / group_size, 2] is wanted")
    _tensor(codes, "codes", device, torch.uint8, (N, K // 2))
    _want(y_dtype in _TYPE, "y_dtype: BF16 or F32 is wanted")
    if out is None:
        out = x.new_empty((T, N)) if y_dtype == BF16 else torch.empty((T, N), dtype=_TYPE[y_dtype], device=device)
    else:
        _tensor(out, "out", device, _TYPE[y_dtype], (T, N))
    _call("dynamo_linear_forward", device, x.data_ptr(), T, N, K, K // groups, codes.data_ptr(), params.data_ptr(),
          out.data_ptr(), y_dtype)
    return out
