"""The calls of include/osscar.h that run, serve, score and train on a pruned layer: gated feed-forward, 8-bit integer products,
log probabilities.  Argument marshalling only, as in binding.py: the outputs and the workspace are torch tensors made here (on
`stream`), everything is computed by the library, and no call waits for the GPU.

Matrices are 2-D tensors on one GPU whose rows are contiguous; weights of a projection are d x f, and may lie in memory that way or as
the transpose of a contiguous f x d tensor.  `stream` defaults to the current stream; tensors made on another stream are the caller's to
order, as everywhere in torch.

Nothing here is recorded by autograd: results never require a gradient, whatever the arguments do, and a loss.backward() that comes to one ends
there.  The gradients of a call are those that its *_backward call returns; to have torch go on from a result, as H.requires_grad_() and
osscar_gated_backward(..., H.grad) do, is the caller's."""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import NamedTuple, Optional, Tuple

import torch

from .binding import OSSCAR_ACT_SILU, OSSCAR_BF16, OSSCAR_F32, OSSCAR_I8, OsscarError, _GatedDesc, load_library

_CODES = {torch.float32: OSSCAR_F32, torch.bfloat16: OSSCAR_BF16}
_EINVAL = 1
_NO_CONTEXT = contextlib.nullcontext()


def _refuse(message: str):
    raise OsscarError(_EINVAL, message)


def _code(t: torch.Tensor, what: str) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        _refuse(f"{what}: dtype {t.dtype} is neither float32 nor bfloat16")
    return code


def _ld(t: torch.Tensor, what: str) -> int:
    """Leading dimension of a matrix with contiguous rows."""
    if t.dim() != 2:
        _refuse(f"{what} must be a matrix")
    rows, cols = t.shape
    s0, s1 = t.stride()
    if cols > 1 and s1 != 1:
        _refuse(f"the rows of {what} must be contiguous")
    if rows <= 1:
        return max(cols, 1)
    if s0 < cols:
        _refuse(f"the rows of {what} overlap")
    return s0


def _on(index: int, **tensors: Optional[torch.Tensor]):
    for name, t in tensors.items():
        if t is not None and t.get_device() != index:
            _refuse(f"{name} is on {t.device}, expected cuda:{index}")


def _vector(t: torch.Tensor, n: int, dtype: torch.dtype, what: str) -> int:
    if t.dim() != 1 or t.shape[0] != n or t.dtype != dtype or (n > 1 and t.stride(0) != 1):
        _refuse(f"{what} must be a contiguous {dtype} vector of {n}")
    return t.data_ptr()


def _begin(t: torch.Tensor, stream: Optional[torch.cuda.Stream]):
    """(library, index of the GPU, stream handle, context in which outputs are made and the call is issued)"""
    index = t.get_device()
    if index < 0:
        _refuse("tensors must be on a GPU")
    if stream is None:
        context = _NO_CONTEXT if index == _current_device() else torch.cuda.device(index)
        return load_library(), index, _current_stream(index), context
    if stream.device.index != index:
        _refuse(f"the stream is on {stream.device}, expected cuda:{index}")
    return load_library(), index, stream.cuda_stream, torch.cuda.stream(stream)


def _current_device() -> int:
    return torch.cuda.current_device()


def _current_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


# The handle without a Stream object around it, where this torch has it: a call of a single token is bound by what the host does.
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", _current_device)
_EMPTY = torch.empty


def _done(lib, status: int):
    if status != 0:
        raise OsscarError(status, lib.osscar_last_error(None).decode())


def _workspace(size: int, device: torch.device):
    """(tensor that holds it or None, its address, its size); the queries add 256 bytes to what is needed, so that 0 says invalid."""
    if size == 0:
        _refuse("invalid sizes")
    if size <= 256:
        return None, None, 0
    ws = _EMPTY(size, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr(), size


def _gated(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, act: int) -> Tuple[_GatedDesc, int, int, int]:
    code = _code(X, "X")
    if X.dim() != 2 or Wg.dim() != 2 or Wg.shape != Wu.shape or Wg.shape[0] != X.shape[1]:
        _refuse("X is n x d, Wg and Wu are d x f")
    if Wg.dtype != X.dtype or Wu.dtype != X.dtype:
        _refuse("X, Wg and Wu have one dtype")
    at = X.get_device()
    if Wg.get_device() != at or Wu.get_device() != at:
        _refuse("X, Wg and Wu are on one GPU")
    n, d = X.shape
    f = Wg.shape[1]
    rows_out = 1 if f > 1 and Wg.stride(1) != 1 else 0
    ldw = _ld(Wg.t() if rows_out else Wg, "Wg")
    if Wg.stride() != Wu.stride() and _ld(Wu.t() if rows_out else Wu, "Wu") != ldw:      # (a dimension of one may have any stride)
        _refuse("Wg and Wu lie in memory alike")
    xp, gp, up = X.data_ptr(), Wg.data_ptr(), Wu.data_ptr()
    return _GatedDesc(n, d, f, _ld(X, "X"), ldw, f, code, act, rows_out, 1 if (xp | gp | up) & 15 else 0), xp, gp, up


def osscar_gated_forward(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, act: int = OSSCAR_ACT_SILU, save: bool = False,
                         stream: Optional[torch.cuda.Stream] = None):
    """H = act(X Wg) * (X Wu).  X: n x d, Wg, Wu: d x f, all float32 or all bfloat16.  save: returns (H, G, U) with the float32 projections
    that osscar_gated_backward takes, else H."""
    lib, index, handle, context = _begin(X, stream)
    desc, xp, gp, up = _gated(X, Wg, Wu, act)
    n, f, device = desc.n, desc.f, X.device
    with context:
        H = _EMPTY(n, f, dtype=X.dtype, device=device)
        G = U = None
        if save:
            G, U = _EMPTY(n, f, dtype=torch.float32, device=device), _EMPTY(n, f, dtype=torch.float32, device=device)
        size = lib.osscar_gated_workspace_bytes(C.byref(desc), 0)
        ws, wp, size = _workspace(size, device)
        status = lib.osscar_gated_forward(C.byref(desc), xp, gp, up, H.data_ptr(), G.data_ptr() if save else None, U.data_ptr() if save else None,
                                          wp, size, handle)
    _done(lib, status)
    return (H, G, U) if save else H


def osscar_gated_backward(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, dH: torch.Tensor, act: int = OSSCAR_ACT_SILU,
                          G: Optional[torch.Tensor] = None, U: Optional[torch.Tensor] = None, need_x: bool = True, need_w: bool = True,
                          dw_dtype: Optional[torch.dtype] = None, stream: Optional[torch.cuda.Stream] = None):
    """(dX, dWg, dWu) of osscar_gated_forward for the gradient dH of H; None for what is not needed.  G, U: from forward's save=True (else they
    are computed again).  The weights' gradients lie in memory as the weights do; dw_dtype: float32 or bfloat16, by default the weights'."""
    lib, index, handle, context = _begin(X, stream)
    desc, xp, gp, up = _gated(X, Wg, Wu, act)
    n, d, f, device = desc.n, desc.d, desc.f, X.device
    if dH.shape != (n, f) or dH.dtype != X.dtype:
        _refuse("dH is n x f, of the dtype of X")
    if (G is None) != (U is None):
        _refuse("G and U are given together or not at all")
    for name, t in (("G", G), ("U", U)):
        if t is not None and (t.shape != (n, f) or t.dtype != torch.float32 or not t.is_contiguous()):
            _refuse(f"{name} must be a contiguous float32 matrix, n x f")
    _on(index, dH=dH, G=G, U=U)
    desc.ldh = _ld(dH, "dH")
    dw_dtype = X.dtype if dw_dtype is None else dw_dtype
    if dw_dtype not in _CODES:
        _refuse(f"dw_dtype {dw_dtype} is neither float32 nor bfloat16")
    with context:
        dX = _EMPTY(n, d, dtype=X.dtype, device=device) if need_x else None
        dWg = dWu = None
        lddw = d if desc.rows_out else f
        if need_w:
            shape = (f, d) if desc.rows_out else (d, f)
            dWg, dWu = _EMPTY(shape, dtype=dw_dtype, device=device), _EMPTY(shape, dtype=dw_dtype, device=device)
        size = lib.osscar_gated_workspace_bytes(C.byref(desc), 1 if G is not None else 2)
        ws, wp, size = _workspace(size, device)
        status = lib.osscar_gated_backward(C.byref(desc), xp, gp, up, dH.data_ptr(), G.data_ptr() if G is not None else None,
                                           U.data_ptr() if U is not None else None, dX.data_ptr() if need_x else None, d,
                                           dWg.data_ptr() if need_w else None, dWu.data_ptr() if need_w else None, lddw, _CODES[dw_dtype], wp,
                                           size, handle)
    _done(lib, status)
    if need_w and desc.rows_out:
        dWg, dWu = dWg.t(), dWu.t()
    return dX, dWg, dWu


def osscar_int_weights(W: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(Wq, w_scale) of W (d1 x m, either layout in memory): Wq is m x ld int8, ld = d1 rounded up to 16, zeros from column d1 on; channel j of W is
    w_scale[j] * Wq[j, :d1] to the nearest."""
    lib, index, handle, context = _begin(W, stream)
    code = _code(W, "W")
    if W.dim() != 2:
        _refuse("W must be a matrix")
    d1, m = W.shape
    rows_out = 1 if m > 1 and W.stride(1) != 1 else 0
    ldw = _ld(W.t() if rows_out else W, "W")
    ldq = -(-d1 // 16) * 16
    with context:
        Wq, scale = _EMPTY(m, ldq, dtype=torch.int8, device=W.device), _EMPTY(m, dtype=torch.float32, device=W.device)
        status = lib.osscar_int_weights(W.data_ptr(), d1, m, ldw, code, rows_out, Wq.data_ptr(), ldq, scale.data_ptr(), handle)
    _done(lib, status)
    return Wq, scale


def osscar_int_rows(X: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(Xq, x_scale) of the rows of X (n x d1), for several products with the same X: Xq is n x d1 int8 (a view of rows padded to 16)."""
    lib, index, handle, context = _begin(X, stream)
    code, ldx = _code(X, "X"), _ld(X, "X")
    n, d1 = X.shape
    ldq = -(-d1 // 16) * 16
    with context:
        Xq, scale = _EMPTY(n, ldq, dtype=torch.int8, device=X.device), _EMPTY(n, dtype=torch.float32, device=X.device)
        status = lib.osscar_int_rows(X.data_ptr(), n, d1, ldx, code, Xq.data_ptr(), ldq, scale.data_ptr(), handle)
    _done(lib, status)
    return Xq[:, :d1], scale


def osscar_int_product(X: torch.Tensor, Wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                       x_scale: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Y = (X quantised row by row) times the weights of osscar_int_weights, n x m.  X: float32 or bfloat16, or int8 with x_scale (osscar_int_rows)."""
    lib, index, handle, context = _begin(X, stream)
    if X.dim() != 2 or Wq.dim() != 2 or Wq.dtype != torch.int8:
        _refuse("X is a matrix, Wq an int8 matrix")
    n, d1 = X.shape
    m = Wq.shape[0]
    if Wq.shape[1] < d1:
        _refuse("Wq has fewer columns than X")
    code = OSSCAR_I8 if X.dtype == torch.int8 else _code(X, "X")
    if (x_scale is not None) != (code == OSSCAR_I8):
        _refuse("x_scale goes with int8 X, and only with it")
    if out_dtype not in _CODES:
        _refuse(f"out_dtype {out_dtype} is neither float32 nor bfloat16")
    device = X.device
    _on(index, Wq=Wq, w_scale=w_scale, bias=bias, x_scale=x_scale)
    wsp = _vector(w_scale, m, torch.float32, "w_scale")
    bp = _vector(bias, m, torch.float32, "bias") if bias is not None else None
    xsp = _vector(x_scale, n, torch.float32, "x_scale") if x_scale is not None else None
    ldx, ldq = _ld(X, "X"), _ld(Wq, "Wq")
    if m == 1 and ldq % 16 and Wq.untyped_storage().nbytes() - Wq.storage_offset() >= -(-d1 // 16) * 16:      # Wq[:, :d1] of one channel
        ldq = -(-d1 // 16) * 16
    with context:
        Y = _EMPTY(n, m, dtype=out_dtype, device=device)
        size = lib.osscar_int_workspace_bytes(n, d1, m)
        ws, wp, size = _workspace(size, device)
        status = lib.osscar_int_product(X.data_ptr(), n, d1, ldx, code, xsp, Wq.data_ptr(), ldq, wsp, m, bp, Y.data_ptr(), m, _CODES[out_dtype],
                                        wp, size, handle)
    _done(lib, status)
    return Y


class LogProbs(NamedTuple):
    """What osscar_logprobs returns.  lse is n x 2: the largest logit m of a row and log sum exp(scale (logits - m))."""
    logp: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor
    top_index: Optional[torch.Tensor]
    top_logp: Optional[torch.Tensor]


def osscar_logprobs(logits: torch.Tensor, targets: torch.Tensor, top: int = 0, scale: float = 1.0,
                    stream: Optional[torch.cuda.Stream] = None) -> LogProbs:
    """Log probability of targets[i] under softmax(scale * logits[i]), the entropy, and the `top` largest logits of every row with their log
    probabilities.  targets: int64, negative where a row has none."""
    lib, index, handle, context = _begin(logits, stream)
    code, ld = _code(logits, "logits"), _ld(logits, "logits")
    n, vocab = logits.shape
    device = logits.device
    _on(index, targets=targets)
    tp = _vector(targets, n, torch.int64, "targets")
    with context:
        out, lse = _EMPTY(2, n, dtype=torch.float32, device=device), _EMPTY(n, 2, dtype=torch.float32, device=device)      # logp and entropy
        top_index = _EMPTY(n, top, dtype=torch.int64, device=device) if top > 0 else None
        top_logp = _EMPTY(n, top, dtype=torch.float32, device=device) if top > 0 else None
        size = lib.osscar_logprobs_workspace_bytes(n, vocab, top)
        ws, wp, size = _workspace(size, device)
        base = out.data_ptr()
        status = lib.osscar_logprobs(logits.data_ptr(), n, vocab, ld, code, tp, scale, top, base, base + 4 * n, lse.data_ptr(),
                                     top_index.data_ptr() if top > 0 else None, top_logp.data_ptr() if top > 0 else None, wp, size, handle)
    _done(lib, status)
    logp, entropy = out.unbind()
    return LogProbs(logp, entropy, lse, top_index, top_logp)


def osscar_logprobs_backward(logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, dlogp: Optional[torch.Tensor] = None,
                             entropy: Optional[torch.Tensor] = None, dentropy: Optional[torch.Tensor] = None,
                             top_index: Optional[torch.Tensor] = None, dtop: Optional[torch.Tensor] = None, scale: float = 1.0,
                             out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Gradient of the logits from those of logp, entropy and top_logp (any may be None).  lse, entropy, top_index: what osscar_logprobs returned
    for these logits and this scale.  out: where to put it, `logits` itself included."""
    lib, index, handle, context = _begin(logits, stream)
    code, ld = _code(logits, "logits"), _ld(logits, "logits")
    n, vocab = logits.shape
    device = logits.device
    _on(index, targets=targets, lse=lse, dlogp=dlogp, entropy=entropy, dentropy=dentropy, top_index=top_index, dtop=dtop, out=out)
    if lse.shape != (n, 2) or lse.dtype != torch.float32 or not lse.is_contiguous():
        _refuse("lse must be the n x 2 float32 tensor of osscar_logprobs")
    if (dtop is None) != (top_index is None) or (dentropy is not None and entropy is None):
        _refuse("dtop goes with top_index, dentropy with entropy")
    top = 0
    if dtop is not None:
        if dtop.dim() != 2 or dtop.shape[0] != n or dtop.shape != top_index.shape or dtop.dtype != torch.float32 or top_index.dtype != torch.int64 \
                or not dtop.is_contiguous() or not top_index.is_contiguous():
            _refuse("top_index (int64) and dtop (float32) must be contiguous and n x top")
        top = dtop.shape[1]
    if out is not None and (out.shape != logits.shape or out.dtype != logits.dtype):
        _refuse("out must have the shape and dtype of logits")
    tp = _vector(targets, n, torch.int64, "targets")
    rows = [None if t is None else _vector(t, n, torch.float32, name) for name, t in (("dlogp", dlogp), ("entropy", entropy), ("dentropy", dentropy))]
    with context:
        if out is None:
            out = _EMPTY(n, vocab, dtype=logits.dtype, device=device)
        status = lib.osscar_logprobs_backward(logits.data_ptr(), n, vocab, ld, code, tp, scale, lse.data_ptr(), rows[0], rows[1], rows[2], top,
                                              top_index.data_ptr() if top > 0 else None, dtop.data_ptr() if top > 0 else None, out.data_ptr(), _ld(out, "out"),
                                              handle)
    _done(lib, status)
    return out
