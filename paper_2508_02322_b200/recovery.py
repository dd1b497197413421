"""ctypes binding of the recovery operators (include/camera.h): the gated feed-forward block of one expert with its
backward pass, log-probabilities of given tokens, distillation from a teacher's top log-probabilities.

Like binding.py: argument marshalling only, every function named as the C entry point it calls.  Tensors a call returns
are allocated on the stream the call runs on.  Outputs have no autograd graph, whatever their inputs require: backward
passes are calls of their own, and write gradients over what their outputs held (sums over micro-batches are the
caller's).
"""
from __future__ import annotations

import ctypes as C
from typing import Dict, Optional, Tuple

import torch

from .binding import CAMERA_BF16, CAMERA_F32, CameraError, _check, alloc_workspace, camera_distill_t, camera_ffn_t, lib

CAMERA_DISTILL_TAIL = 1
CAMERA_MAX_TOP = 128
_F32, _BF16 = torch.float32, torch.bfloat16
_DTYPE = {torch.bfloat16: CAMERA_BF16, torch.float32: CAMERA_F32}


# The current stream's handle; the same as torch.cuda.current_stream(device).cuda_stream without building a Stream
# object, which takes longer than a small kernel.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _enqueue(fn, t: torch.Tensor, *args) -> None:
    """The C call `fn` on the device of t, whichever device is current, and on that device's current stream."""
    device = t.get_device()
    if device == _current_device():
        status = fn(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            status = fn(*args, _raw_stream(device))
    if status:
        _check(status, fn.__name__)


def _elsewhere(stream: Optional[torch.cuda.Stream], fn, *args, **kw):
    """The call with `stream` as the current one, so that what it allocates belongs there."""
    with torch.cuda.stream(stream):
        return fn(*args, **kw)


def _rows(t: torch.Tensor, name: str) -> int:
    """Distance of the rows of a [n_rows, vocab] tensor in elements."""
    if not (t.is_cuda and t.dim() == 2 and t.dtype in _DTYPE):
        raise ValueError(f"{name} must be a bf16 or fp32 [n_rows, vocab] tensor on the GPU")
    rows, vocab = t.shape
    ld, one = t.stride()
    if rows <= 1 and ld < vocab:
        ld = vocab
    if (one != 1 and vocab > 1) or ld < vocab:
        raise ValueError(f"{name} must have contiguous, non-overlapping rows")
    return ld


def _vector(t: torch.Tensor, like: torch.Tensor, dtype, shape, name: str) -> int:
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.device != like.device:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on the device of the logits")
    return t.data_ptr()


class Ffn:
    """Holds the matrices of one gated feed-forward block and the camera_ffn_t that points at them.

    w_gate, w_up: [d_ff, d_model]; w_down: [d_model, down_ld] with down_ld >= d_ff (an expert that camera_compact_weights
    sliced into a buffer of the original width; d_ff then says how many of its columns, and of the rows of w_gate and
    w_up, are in use).
    """

    def __init__(self, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, d_ff: Optional[int] = None):
        f = int(w_gate.shape[0]) if d_ff is None else int(d_ff)
        for t in (w_gate, w_up, w_down):
            if not (t.dim() == 2 and t.is_contiguous() and t.dtype == torch.bfloat16 and t.device == w_gate.device):
                raise ValueError("w_gate, w_up and w_down must be contiguous bf16 matrices on one device")
        d = int(w_gate.shape[1])
        if w_up.shape[1] != d or w_down.shape[0] != d or min(w_gate.shape[0], w_up.shape[0], w_down.shape[1]) < f or f < 1:
            raise ValueError("w_gate and w_up must be [>= d_ff, d_model], w_down [d_model, >= d_ff]")
        self.w_gate, self.w_up, self.w_down = w_gate, w_up, w_down
        self.d_model, self.d_ff, self.down_ld = d, f, int(w_down.shape[1])
        self.device = w_gate.device
        self.c = camera_ffn_t(d, f, self.down_ld, w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr())
        self._ref = C.byref(self.c)
        self._saved_bytes: Dict[int, int] = {}


def camera_ffn_workspace_bytes(ffn: Ffn, n_tokens: int, *, backward: bool = False) -> int:
    n = int(lib.camera_ffn_workspace_bytes(ffn._ref, n_tokens, int(backward)))
    if n == 0:
        raise CameraError(-2, "camera_ffn_workspace_bytes")
    return n


def camera_ffn_saved_bytes(ffn: Ffn, n_tokens: int) -> int:
    n = ffn._saved_bytes.get(n_tokens)
    if n is None:
        n = ffn._saved_bytes[n_tokens] = int(lib.camera_ffn_saved_bytes(ffn._ref, n_tokens))
    return n


def _tokens(t: torch.Tensor, ffn: Ffn, name: str) -> int:
    if t.dtype is not _BF16 or t.dim() != 2 or t.shape[1] != ffn.d_model or not t.is_contiguous() or t.device != ffn.device:
        raise ValueError(f"{name} must be a contiguous bf16 [n_tokens, d_model] tensor on the device of the block")
    if not t.is_cuda:
        raise ValueError(f"the block and {name} must be on a GPU")
    return t.data_ptr()


def _saved(saved: torch.Tensor, ffn: Ffn, n_tokens: int) -> int:
    if saved.numel() * saved.element_size() < camera_ffn_saved_bytes(ffn, n_tokens) or saved.device != ffn.device or \
            not saved.is_contiguous():
        raise ValueError("saved must have camera_ffn_saved_bytes contiguous bytes on the device of the block")
    return saved.data_ptr()


def _workspace(workspace: Optional[torch.Tensor], ffn: Ffn, n_tokens: int, backward: bool) -> torch.Tensor:
    if workspace is None:
        return alloc_workspace(camera_ffn_workspace_bytes(ffn, n_tokens, backward=backward), ffn.device)
    if workspace.device != ffn.device or not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous, on the device of the block")
    return workspace


def camera_ffn_forward(ffn: Ffn, x: torch.Tensor, *, y: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """y = (SiLU(x W_gate^T) * (x W_up^T)) W_down^T, bf16 [n_tokens, d_model].  `saved` (camera_ffn_saved_bytes bytes)
    receives what camera_ffn_backward needs."""
    if stream is not None:
        return _elsewhere(stream, camera_ffn_forward, ffn, x, y=y, saved=saved, workspace=workspace)
    xp = _tokens(x, ffn, "x")
    n = x.shape[0]
    if y is None:
        y = torch.empty_like(x)
    elif _tokens(y, ffn, "y") is None or y.shape[0] != n:
        raise ValueError("y must have the shape of x")
    workspace = _workspace(workspace, ffn, n, False)
    _enqueue(lib.camera_ffn_forward, x, ffn._ref, xp, n, y.data_ptr(), None if saved is None else _saved(saved, ffn, n),
             workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return y


def camera_ffn_backward(ffn: Ffn, x: torch.Tensor, dy: torch.Tensor, saved: torch.Tensor, *, want_x: bool = True,
                        want_weights: bool = True, out: Optional[Dict[str, torch.Tensor]] = None,
                        workspace: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """Gradients of camera_ffn_forward(ffn, x, saved=saved) given dy: a dict with x (want_x) and w_gate, w_up [d_ff,
    d_model], w_down [d_model, down_ld] (want_weights; columns of w_down from d_ff on are not written).  `out` names
    tensors of those shapes to write to."""
    if stream is not None:
        return _elsewhere(stream, camera_ffn_backward, ffn, x, dy, saved, want_x=want_x, want_weights=want_weights, out=out,
                          workspace=workspace)
    xp, dyp = _tokens(x, ffn, "x"), _tokens(dy, ffn, "dy")
    n, f, d = x.shape[0], ffn.d_ff, ffn.d_model
    if dy.shape[0] != n:
        raise ValueError("dy must have the shape of x")
    sp = _saved(saved, ffn, n)
    res: Dict[str, torch.Tensor] = {}
    ptr = [None, None, None, None]
    for i, (name, rows, cols, want) in enumerate((("x", n, d, want_x), ("w_gate", f, d, want_weights),
                                                  ("w_up", f, d, want_weights), ("w_down", d, ffn.down_ld, want_weights))):
        if not want:
            continue
        t = out.get(name) if out else None
        if t is None:
            t = torch.empty((rows, cols), dtype=_BF16, device=ffn.device)
        elif t.dtype is not _BF16 or t.shape != (rows, cols) or not t.is_contiguous() or t.device != ffn.device:
            raise ValueError(f"out[{name!r}] must be a contiguous bf16 tensor of shape {(rows, cols)}")
        res[name] = t
        ptr[i] = t.data_ptr()
    workspace = _workspace(workspace, ffn, n, True)
    _enqueue(lib.camera_ffn_backward, x, ffn._ref, xp, dyp, n, sp, ptr[0], ptr[1], ptr[2], ptr[3], workspace.data_ptr(),
             workspace.numel() * workspace.element_size())
    return res


def camera_token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, *, top_n: int = 0,
                          temperature: float = 1.0, entropy: bool = True,
                          stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """Log-probability of targets[r] (int64 [n_rows]) under softmax(logits[r] / temperature), the entropy of that
    distribution, and its top_n alternatives.  Returns a dict with logprob (if targets are given), entropy (unless
    entropy=False), and for top_n > 0 top_idx (int32) and top_logprob [n_rows, top_n]."""
    if stream is not None:
        return _elsewhere(stream, camera_token_logprobs, logits, targets, top_n=top_n, temperature=temperature, entropy=entropy)
    ld = _rows(logits, "logits")
    rows, vocab = logits.shape
    out: Dict[str, torch.Tensor] = {}
    dev = logits.device
    t_ptr = lp_ptr = h_ptr = i_ptr = v_ptr = None
    if targets is not None:
        t_ptr = _vector(targets, logits, torch.int64, (rows,), "targets")
        out["logprob"] = t = torch.empty(rows, dtype=_F32, device=dev)
        lp_ptr = t.data_ptr()
    if entropy:
        out["entropy"] = t = torch.empty(rows, dtype=_F32, device=dev)
        h_ptr = t.data_ptr()
    if top_n > 0:
        out["top_idx"] = t = torch.empty(rows, top_n, dtype=torch.int32, device=dev)
        i_ptr = t.data_ptr()
        out["top_logprob"] = t = torch.empty(rows, top_n, dtype=_F32, device=dev)
        v_ptr = t.data_ptr()
    _enqueue(lib.camera_token_logprobs, logits, logits.data_ptr(), _DTYPE[logits.dtype], ld, rows, vocab, t_ptr, top_n, temperature,
             lp_ptr, h_ptr, i_ptr, v_ptr)
    return out


def _distill(logits, teacher_idx, teacher_logprob, temperature, tail) -> camera_distill_t:
    ld = _rows(logits, "logits")
    rows, vocab = logits.shape
    if teacher_idx.dim() != 2:
        raise ValueError("teacher_idx must be [n_rows, k]")
    k = int(teacher_idx.shape[1])
    return camera_distill_t(logits.data_ptr(), ld, rows, _DTYPE[logits.dtype], vocab,
                            _vector(teacher_idx, logits, torch.int32, (rows, k), "teacher_idx"),
                            _vector(teacher_logprob, logits, torch.float32, (rows, k), "teacher_logprob"), k, temperature,
                            CAMERA_DISTILL_TAIL if tail else 0)


def _gradient(logits: torch.Tensor, d_logits: Optional[torch.Tensor], ld: int) -> Tuple[torch.Tensor, int]:
    """The gradient's tensor and its pitch: where it is allocated, the vocabulary and what aligns its rows to 16 bytes as
    those of the logits are, however far apart they lie."""
    if d_logits is None:
        vocab = logits.shape[1]
        ld = vocab + (ld - vocab) % (16 // logits.element_size())
        return torch.empty_strided(logits.shape, (ld, 1), dtype=logits.dtype, device=logits.device), ld
    if d_logits.shape != logits.shape or d_logits.dtype != logits.dtype or d_logits.device != logits.device:
        raise ValueError("d_logits must have the shape, dtype and device of the logits")
    return d_logits, _rows(d_logits, "d_logits")


def camera_distill_forward(logits: torch.Tensor, teacher_idx: torch.Tensor, teacher_logprob: torch.Tensor, *,
                           temperature: float = 1.0, tail: bool = False,
                           stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """Divergence of the student (softmax(logits / temperature)) from the teacher's list (int32 / fp32 [n_rows, k], as
    camera_token_logprobs returns them) per row.  Returns a dict with loss [n_rows] and what camera_distill_backward
    takes: lse and, with tail=True (the rest of the vocabulary as one more class), log_tail."""
    if stream is not None:
        return _elsewhere(stream, camera_distill_forward, logits, teacher_idx, teacher_logprob, temperature=temperature, tail=tail)
    d = _distill(logits, teacher_idx, teacher_logprob, temperature, tail)
    out = {name: torch.empty(d.n_rows, dtype=_F32, device=logits.device)
           for name in (("loss", "lse", "log_tail") if tail else ("loss", "lse"))}
    _enqueue(lib.camera_distill_forward, logits, C.byref(d), out["loss"].data_ptr(), out["lse"].data_ptr(),
             out["log_tail"].data_ptr() if tail else None)
    return out


def camera_distill_backward(logits: torch.Tensor, teacher_idx: torch.Tensor, teacher_logprob: torch.Tensor,
                            d_loss: torch.Tensor, lse: torch.Tensor, log_tail: Optional[torch.Tensor] = None, *,
                            temperature: float = 1.0, tail: bool = False,
                            d_logits: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Gradient by the logits, d_loss [n_rows] being the gradient by the losses; lse and log_tail are the forward
    call's.  d_logits may be the logits themselves."""
    if stream is not None:
        return _elsewhere(stream, camera_distill_backward, logits, teacher_idx, teacher_logprob, d_loss, lse, log_tail,
                          temperature=temperature, tail=tail, d_logits=d_logits)
    d = _distill(logits, teacher_idx, teacher_logprob, temperature, tail)
    rows = (d.n_rows,)
    if tail and log_tail is None:
        raise ValueError("log_tail is needed with tail=True")
    d_logits, d_ld = _gradient(logits, d_logits, d.ld)
    _enqueue(lib.camera_distill_backward, logits, C.byref(d), _vector(d_loss, logits, torch.float32, rows, "d_loss"),
             _vector(lse, logits, torch.float32, rows, "lse"),
             _vector(log_tail, logits, torch.float32, rows, "log_tail") if tail else None, d_logits.data_ptr(), d_ld)
    return d_logits


def camera_distill_step(logits: torch.Tensor, teacher_idx: torch.Tensor, teacher_logprob: torch.Tensor,
                        d_loss: torch.Tensor, *, temperature: float = 1.0, tail: bool = False,
                        d_logits: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Loss and gradient from one call, for a d_loss known beforehand.  Returns (loss, d_logits)."""
    if stream is not None:
        return _elsewhere(stream, camera_distill_step, logits, teacher_idx, teacher_logprob, d_loss, temperature=temperature,
                          tail=tail, d_logits=d_logits)
    d = _distill(logits, teacher_idx, teacher_logprob, temperature, tail)
    d_logits, d_ld = _gradient(logits, d_logits, d.ld)
    loss = torch.empty(d.n_rows, dtype=_F32, device=logits.device)
    _enqueue(lib.camera_distill_step, logits, C.byref(d), _vector(d_loss, logits, torch.float32, (d.n_rows,), "d_loss"),
             loss.data_ptr(), d_logits.data_ptr(), d_ld)
    return loss, d_logits
