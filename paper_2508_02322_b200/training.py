"""ctypes binding of the operators around a layer's experts when the layer is trained (include/camera.h): norms with their
backward pass, tokens sorted by expert and back with the gradients of both, orthogonalised updates.

Like recovery.py: argument marshalling only, every function named as the C entry point it calls; tensors a call returns are
allocated on the stream the call runs on; outputs have no autograd graph.
"""
from __future__ import annotations

import ctypes as C
from typing import Dict, List, Optional, Sequence, Tuple, Union

import torch

from .binding import CAMERA_BF16, CAMERA_F32, CameraError, alloc_workspace, camera_matrix_t, camera_norm_t, lib
from .recovery import _elsewhere, _enqueue

CAMERA_NORM_RMS = 1
# (a, b, c) of a s + b s^3 + c s^5, applied five times: takes singular values of [0.003, 1] into about [0.7, 1.2]
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)
_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32
_DTYPE = {torch.bfloat16: CAMERA_BF16, torch.float32: CAMERA_F32}


def _matrix(t: torch.Tensor, name: str, like: Optional[torch.Tensor] = None, rows: Optional[int] = None,
            cols: Optional[int] = None) -> int:
    """Distance of the rows of a [rows, cols] matrix in elements; like: whose dtype and device it shares."""
    if like is not None:
        if t.dtype is not like.dtype or t.get_device() != like.get_device():
            raise ValueError(f"{name} must have the dtype and device of the other matrices of the call")
    elif not t.is_cuda or t.dtype not in _DTYPE:
        raise ValueError(f"{name} must be a bf16 or fp32 matrix on the GPU")
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix")
    r, c = t.shape
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise ValueError(f"{name} must have the shape {(rows if rows is not None else r, cols if cols is not None else c)}")
    ld, one = t.stride()
    if ld < c or one != 1:
        if r <= 1 and ld < c:
            ld = c
        if (one != 1 and c > 1) or ld < c:
            raise ValueError(f"{name} must have contiguous, non-overlapping rows")
    return ld


def _result(like: torch.Tensor, rows: int, cols: int) -> Tuple[torch.Tensor, int]:
    """A new matrix of the dtype and device of `like`, and the distance of its rows."""
    return like.new_empty((rows, cols)), cols


def _array(t: torch.Tensor, like: torch.Tensor, dtype, shape, name: str) -> int:
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != like.get_device():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the device of the matrices")
    return t.data_ptr()


def _scratch(workspace: Optional[torch.Tensor], nbytes, device) -> torch.Tensor:
    if workspace is None:
        return alloc_workspace(nbytes(), device)
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous, on the device of the matrices")
    return workspace


# ------------------------------------------------------------------------------------------------ norms
def _norm(x, weight, bias, eps, rms) -> camera_norm_t:
    ld = _matrix(x, "x")
    rows, d = x.shape
    wp = bp = None
    wt = _DTYPE[x.dtype]
    for name, t in (("weight", weight), ("bias", bias)):
        if t is None:
            continue
        if t.dtype not in _DTYPE or t.shape != (d,) or not t.is_contiguous() or t.device != x.device:
            raise ValueError(f"{name} must be a contiguous bf16 or fp32 tensor of shape {(d,)} on the device of x")
        wt = _DTYPE[t.dtype]
        if name == "weight":
            wp = t.data_ptr()
        else:
            bp = t.data_ptr()
    if weight is not None and bias is not None and weight.dtype is not bias.dtype:
        raise ValueError("weight and bias must have the same dtype")
    return camera_norm_t(x.data_ptr(), ld, rows, _DTYPE[x.dtype], d, wp, bp, wt, eps, CAMERA_NORM_RMS if rms else 0)


def camera_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
                        residual: Optional[torch.Tensor] = None, eps: float = 1e-6, rms: bool = False, stats: bool = True,
                        out: Optional[Dict[str, torch.Tensor]] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """Layer norm of the rows of x + residual (rms=True: root mean square norm), times weight, plus bias.  Returns a dict
    with y, with sum (x + residual) where there is a residual, and, for camera_norm_backward (stats=False leaves them out),
    rstd and (unless rms) mean, fp32 [n_rows].  `out` names tensors to write y and sum to; both may be x or residual."""
    if stream is not None:
        return _elsewhere(stream, camera_norm_forward, x, weight, bias, residual=residual, eps=eps, rms=rms, stats=stats, out=out)
    for name in out or ():
        if out[name] is not None and name != "y" and (name != "sum" or residual is None):
            raise ValueError(f"out names y and, with a residual, sum: not {name}")
    n = _norm(x, weight, bias, eps, rms)
    rows, d = x.shape
    y = out.get("y") if out else None
    y, y_ld = _result(x, rows, d) if y is None else (y, _matrix(y, "out['y']", x, rows, d))
    res: Dict[str, torch.Tensor] = {"y": y}
    r_ptr = z_ptr = m_ptr = s_ptr = None
    r_ld = z_ld = 0
    if residual is not None:
        r_ptr, r_ld = residual.data_ptr(), _matrix(residual, "residual", x, rows, d)
        z = out.get("sum") if out else None
        z, z_ld = _result(x, rows, d) if z is None else (z, _matrix(z, "out['sum']", x, rows, d))
        z_ptr = z.data_ptr()
        res["sum"] = z
    if stats:
        if not rms:
            res["mean"] = t = x.new_empty(rows, dtype=_F32)
            m_ptr = t.data_ptr()
        res["rstd"] = t = x.new_empty(rows, dtype=_F32)
        s_ptr = t.data_ptr()
    _enqueue(lib.camera_norm_forward, x, C.byref(n), r_ptr, r_ld, z_ptr, z_ld, y.data_ptr(), y_ld, m_ptr, s_ptr)
    return res


def camera_norm_backward_workspace_bytes(n_rows: int, d: int) -> int:
    n = int(lib.camera_norm_backward_workspace_bytes(n_rows, d))
    if n == 0:
        raise CameraError(-2, "camera_norm_backward_workspace_bytes")
    return n


def camera_norm_backward(dy: torch.Tensor, x: torch.Tensor, rstd: torch.Tensor, mean: Optional[torch.Tensor] = None,
                         weight: Optional[torch.Tensor] = None, *, d_sum: Optional[torch.Tensor] = None, want_x: bool = True,
                         want_weight: bool = True, want_bias: bool = False, out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """Gradients of camera_norm_forward given dy.  x is what was normalised (the forward call's `sum` where there was a
    residual), rstd and mean are that call's; no mean: a root mean square norm.  d_sum: the gradient that reaches x (or sum)
    from elsewhere, added to dx.  Returns a dict with x (the residual's gradient too), weight and bias (fp32 [d]) as asked
    for.  `out`: where dx goes; may be dy, d_sum or x."""
    if stream is not None:
        return _elsewhere(stream, camera_norm_backward, dy, x, rstd, mean, weight, d_sum=d_sum, want_x=want_x,
                          want_weight=want_weight, want_bias=want_bias, out=out, workspace=workspace)
    if not want_x and out is not None:
        raise ValueError("out belongs to the gradient of x: not with want_x=False")
    n = _norm(x, weight, None, 0.0, mean is None)
    rows, d = x.shape
    dy_ld = _matrix(dy, "dy", x, rows, d)
    s_ptr = _array(rstd, x, _F32, (rows,), "rstd")
    m_ptr = None if mean is None else _array(mean, x, _F32, (rows,), "mean")
    z_ptr, z_ld = (None, 0) if d_sum is None else (d_sum.data_ptr(), _matrix(d_sum, "d_sum", x, rows, d))
    res: Dict[str, torch.Tensor] = {}
    dx_ptr, dx_ld, w_ptr, b_ptr, ws_ptr, ws_n = None, 0, None, None, None, 0
    if want_x:
        out, dx_ld = _result(x, rows, d) if out is None else (out, _matrix(out, "out", x, rows, d))
        res["x"], dx_ptr = out, out.data_ptr()
    if want_weight:
        res["weight"] = t = x.new_empty(d, dtype=_F32)
        w_ptr = t.data_ptr()
    if want_bias:
        res["bias"] = t = x.new_empty(d, dtype=_F32)
        b_ptr = t.data_ptr()
    if want_weight or want_bias:
        workspace = _scratch(workspace, lambda: camera_norm_backward_workspace_bytes(rows, d), x.device)
        ws_ptr, ws_n = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _enqueue(lib.camera_norm_backward, x, C.byref(n), dy.data_ptr(), dy_ld, m_ptr, s_ptr, z_ptr, z_ld, dx_ptr, dx_ld, w_ptr, b_ptr,
             ws_ptr, ws_n)
    return res


# ------------------------------------------------------------------------------------------------ tokens to experts and back
def _pairs(t: torch.Tensor, dtype, like: torch.Tensor, name: str) -> Tuple[int, int]:
    if t.dtype is not dtype or t.dim() != 2 or t.shape[1] < 1 or not t.is_contiguous() or t.get_device() != like.get_device():
        raise ValueError(f"{name} must be a contiguous {dtype} [n_tokens, top_k] tensor on the device of the matrices")
    return t.shape


def camera_moe_dispatch_workspace_bytes(n_tokens: int, top_k: int, n_experts: int) -> int:
    n = int(lib.camera_moe_dispatch_workspace_bytes(n_tokens, top_k, n_experts))
    if n == 0:
        raise CameraError(-2, "camera_moe_dispatch_workspace_bytes")
    return n


def camera_moe_dispatch(x: torch.Tensor, topk_idx: torch.Tensor, n_experts: int, *, out: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """Rows of x [n_tokens, d_model] copied to the experts that topk_idx (int32 [n_tokens, top_k], as camera_score_layer's
    details hold it) names, sorted by expert.  Returns a dict with x [n_tokens * top_k, d_model], rows (int32 [n_tokens,
    top_k]: where each pair went, -1 for an index outside [0, n_experts)) and offsets (int32 [n_experts + 1]).  `out`: a
    matrix of at least as many rows to write x to; rows from offsets[n_experts] on are not written."""
    if stream is not None:
        return _elsewhere(stream, camera_moe_dispatch, x, topk_idx, n_experts, out=out, workspace=workspace)
    ld = _matrix(x, "x")
    tokens, d = x.shape
    t, k = _pairs(topk_idx, _I32, x, "topk_idx")
    if t != tokens:
        raise ValueError("topk_idx must have a row for each token")
    if out is None:
        out, out_ld = _result(x, tokens * k, d)
    else:
        out_ld = _matrix(out, "out", x, None, d)
        if out.shape[0] < tokens * k:
            raise ValueError("out must have room for n_tokens * top_k rows")
    rows = topk_idx.new_empty((tokens, k))
    offsets = topk_idx.new_empty(max(int(n_experts), 0) + 1)
    workspace = _scratch(workspace, lambda: camera_moe_dispatch_workspace_bytes(tokens, k, n_experts), x.device)
    _enqueue(lib.camera_moe_dispatch, x, x.data_ptr(), _DTYPE[x.dtype], ld, tokens, d, topk_idx.data_ptr(), k, n_experts,
             out.data_ptr(), out_ld, rows.data_ptr(), offsets.data_ptr(), workspace.data_ptr(),
             workspace.numel() * workspace.element_size())
    return {"x": out, "rows": rows, "offsets": offsets}


def _back(fn, sorted_rows, rows, topk_w, add, out):
    ld = _matrix(sorted_rows, "the sorted rows")
    n, d = sorted_rows.shape
    tokens, k = _pairs(rows, _I32, sorted_rows, "rows")
    w = () if fn is lib.camera_moe_dispatch_backward else \
        (None if topk_w is None else _array(topk_w, sorted_rows, _F32, (tokens, k), "topk_w"),)
    a_ptr, a_ld = (None, 0) if add is None else (add.data_ptr(), _matrix(add, "add", sorted_rows, tokens, d))
    out, out_ld = _result(sorted_rows, tokens, d) if out is None else (out, _matrix(out, "out", sorted_rows, tokens, d))
    _enqueue(fn, sorted_rows, sorted_rows.data_ptr(), _DTYPE[sorted_rows.dtype], ld, n, rows.data_ptr(), *w, tokens, k, d, a_ptr,
             a_ld, out.data_ptr(), out_ld)
    return out


def camera_moe_combine(y_sorted: torch.Tensor, rows: torch.Tensor, topk_w: Optional[torch.Tensor] = None, *,
                       add: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """y[t] = add[t] + sum over the slots of topk_w[t, j] y_sorted[rows[t, j]] (no topk_w: ones), [n_tokens, d_model] in the
    dtype of y_sorted; rows as camera_moe_dispatch returned them.  `out` may be add."""
    if stream is not None:
        return _elsewhere(stream, camera_moe_combine, y_sorted, rows, topk_w, add=add, out=out)
    return _back(lib.camera_moe_combine, y_sorted, rows, topk_w, add, out)


def camera_moe_dispatch_backward(dx_sorted: torch.Tensor, rows: torch.Tensor, *, add: Optional[torch.Tensor] = None,
                                 out: Optional[torch.Tensor] = None,
                                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Gradient of camera_moe_dispatch by its tokens: add[t] + sum over the slots of dx_sorted[rows[t, j]]."""
    if stream is not None:
        return _elsewhere(stream, camera_moe_dispatch_backward, dx_sorted, rows, add=add, out=out)
    return _back(lib.camera_moe_dispatch_backward, dx_sorted, rows, None, add, out)


def camera_moe_combine_backward(dy: torch.Tensor, y_sorted: torch.Tensor, rows: torch.Tensor,
                                topk_w: Optional[torch.Tensor] = None, *, want_y: bool = True, want_weights: bool = True,
                                out: Optional[torch.Tensor] = None,
                                stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """Gradients of camera_moe_combine given dy [n_tokens, d_model]: a dict with y (of y_sorted's shape; rows that no pair
    names are not written) and weights (fp32 [n_tokens, top_k]).  add's gradient is dy.  `out`: where y goes; may be
    y_sorted."""
    if stream is not None:
        return _elsewhere(stream, camera_moe_combine_backward, dy, y_sorted, rows, topk_w, want_y=want_y,
                          want_weights=want_weights, out=out)
    if not want_y and out is not None:
        raise ValueError("out belongs to the gradient of y_sorted: not with want_y=False")
    ld = _matrix(dy, "dy")
    tokens, d = dy.shape
    ys_ld = _matrix(y_sorted, "y_sorted", dy, None, d)
    n = y_sorted.shape[0]
    t, k = _pairs(rows, _I32, dy, "rows")
    if t != tokens:
        raise ValueError("rows must have a row for each token")
    w_ptr = None if topk_w is None else _array(topk_w, dy, _F32, (tokens, k), "topk_w")
    res: Dict[str, torch.Tensor] = {}
    o_ptr, o_ld, dw_ptr = None, 0, None
    if want_y:
        out, o_ld = _result(dy, n, d) if out is None else (out, _matrix(out, "out", dy, n, d))
        res["y"], o_ptr = out, out.data_ptr()
    if want_weights:
        res["weights"] = w = dy.new_empty((tokens, k), dtype=_F32)
        dw_ptr = w.data_ptr()
    _enqueue(lib.camera_moe_combine_backward, dy, dy.data_ptr(), _DTYPE[dy.dtype], ld, tokens, d, rows.data_ptr(), w_ptr, k,
             y_sorted.data_ptr(), ys_ld, n, o_ptr, o_ld, dw_ptr)
    return res


# ------------------------------------------------------------------------------------------------ orthogonalised updates
Updates = Union[torch.Tensor, Sequence[torch.Tensor]]


def _list(updates: Updates) -> List[torch.Tensor]:
    if isinstance(updates, torch.Tensor):
        if updates.dim() != 3:
            raise ValueError("updates must be a list of matrices or a tensor [n, rows, cols]")
        return list(updates.unbind(0))
    return list(updates)


def camera_orthogonalize_workspace_bytes(updates: Updates) -> int:
    mats = _list(updates)
    arr = (camera_matrix_t * len(mats))(*[camera_matrix_t(None, None, 0, 0, *t.shape) for t in mats])
    n = int(lib.camera_orthogonalize_workspace_bytes(arr, len(mats)))
    if n == 0:
        raise CameraError(-2, "camera_orthogonalize_workspace_bytes")
    return n


def camera_orthogonalize(updates: Updates, *, steps: Optional[int] = None, coefficients=NEWTON_SCHULZ, eps: float = 1e-7,
                         out: Optional[Updates] = None, workspace: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> Updates:
    """The matrices of `updates` (bf16 or fp32, a list of any shapes or a tensor [n, rows, cols]), each over its norm (plus
    eps) and with every singular value s taken to a s + b s^3 + c s^5, `steps` times over (5 if not given).  coefficients:
    (a, b, c), or a list of such for each step, as many as there are steps.  Returns bf16 matrices of the same shapes (`out`,
    if given; may be bf16 updates themselves)."""
    if stream is not None:
        return _elsewhere(stream, camera_orthogonalize, updates, steps=steps, coefficients=coefficients, eps=eps, out=out,
                          workspace=workspace)
    mats = _list(updates)
    one = len(coefficients) == 3 and not any(isinstance(c, (tuple, list)) for c in coefficients)
    each = [tuple(coefficients)] * (5 if steps is None else steps) if one else coefficients
    if not each or not all(isinstance(c, (tuple, list)) and len(c) == 3 for c in each):
        raise ValueError("coefficients must be three numbers, or three for each step")
    if steps is not None and len(each) != steps:
        raise ValueError(f"coefficients of {len(each)} steps, and steps = {steps}")
    flat = [float(v) for c in each for v in c]
    if out is None:
        out = torch.empty(updates.shape, dtype=_BF16, device=updates.device) if isinstance(updates, torch.Tensor) else \
            [torch.empty(t.shape, dtype=_BF16, device=t.device) for t in mats]
    outs = _list(out)
    if not mats:
        return out
    if len(outs) != len(mats):
        raise ValueError("out must have a matrix for each update")
    arr = (camera_matrix_t * len(mats))()
    for a, t, o in zip(arr, mats, outs):
        a.in_ld, a.out_ld = _matrix(t, "an update", mats[0]), _matrix(o, "out", None, *t.shape)
        if o.dtype is not _BF16 or o.device != t.device:
            raise ValueError("out must be bf16, on the device of the updates")
        a.in_, a.out = t.data_ptr(), o.data_ptr()
        a.rows, a.cols = t.shape
    workspace = _scratch(workspace, lambda: camera_orthogonalize_workspace_bytes(mats), mats[0].device)
    _enqueue(lib.camera_orthogonalize, mats[0], arr, len(mats), _DTYPE[mats[0].dtype], (C.c_float * len(flat))(*flat), len(flat) // 3,
             eps, workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return out
