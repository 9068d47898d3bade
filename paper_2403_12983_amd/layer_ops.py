"""The calls of include/osscar.h that run, serve, score, repair and train on a pruned layer: gated feed-forward, 8-bit integer products,
log probabilities, layer norm, low-rank adapters, AdamW.  Argument marshalling only, as in binding.py: the outputs and the workspace are torch tensors made here (on
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
import math
from typing import List, NamedTuple, Optional, Sequence, Tuple, Union

import torch

from .binding import OSSCAR_ACT_SILU, OSSCAR_BF16, OSSCAR_F32, OSSCAR_I8, OsscarError, _AdamWDesc, _AdamWTensor, _AdaptersDesc, _GatedDesc, load_library, load_tensors

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


def _on(index: int, /, **tensors: Optional[torch.Tensor]):
    for name, t in tensors.items():
        if t is not None and t.get_device() != index:
            _refuse(f"{name} is on {t.device}, expected cuda:{index}")


def _vector(t: torch.Tensor, n: int, dtype: torch.dtype, what: str) -> int:
    if t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
        _refuse(f"{what} must be a contiguous {dtype} vector of {n}")
    return t.data_ptr()


def _vector_on(index: int, t: torch.Tensor, n: int, dtype: torch.dtype, what: str) -> int:
    if t.get_device() != index:
        _refuse(f"{what} is on {t.device}, expected cuda:{index}")
    return _vector(t, n, dtype, what)


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


def _out(out: Optional[torch.Tensor], like: torch.Tensor, shape) -> torch.Tensor:
    if out is None:
        return _EMPTY(shape, dtype=like.dtype, device=like.device)
    if out.shape != shape or out.dtype != like.dtype:
        _refuse("out has another shape or dtype than the result")
    return out


def _gains(index: int, w: Optional[torch.Tensor], d: int, what: str) -> Tuple[Optional[int], Optional[int]]:
    """(address, dtype) of a vector over the columns, or of none"""
    return (None, None) if w is None else (_vector_on(index, w, d, w.dtype, what), _code(w, what))


def osscar_layernorm_forward(X: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, save: bool = False,
                             out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Layer norm of the rows of X (n x d): (x - mean) / sqrt(var + eps) * weight + bias.  weight, bias: d, float32 or bfloat16 (both the same), or None.  save: returns
    (Y, stats) with the mean and 1 / sqrt(var + eps) of each row that osscar_layernorm_backward takes, else Y.  out: where to put Y, `X` itself included."""
    lib, index, handle, context = _begin(X, stream)
    code, ldx = _code(X, "X"), _ld(X, "X")
    n, d = X.shape
    if out is not None:
        _on(index, out=out)
    (wp, wc), (bp, bc) = _gains(index, weight, d, "weight"), _gains(index, bias, d, "bias")
    if wc is not None and bc is not None and wc != bc:
        _refuse("weight and bias have one dtype")
    with context:
        Y = _out(out, X, X.shape)
        stats = _EMPTY(n, 2, dtype=torch.float32, device=X.device) if save else None
        status = lib.osscar_layernorm_forward(X.data_ptr(), n, d, ldx, code, wp, bp, wc if wc is not None else bc if bc is not None else code, eps, Y.data_ptr(),
                                              _ld(Y, "out"), stats.data_ptr() if save else None, handle)
    _done(lib, status)
    return (Y, stats) if save else Y


def osscar_layernorm_backward(X: torch.Tensor, weight: Optional[torch.Tensor], dY: torch.Tensor, stats: torch.Tensor, need_x: bool = True, need_w: bool = True,
                              dw_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """(dX, dweight, dbias) of osscar_layernorm_forward for the gradient dY of Y; None for what is not needed.  stats: from forward's save=True.  dw_dtype: float32 or bfloat16,
    by default the weight's (without one: that of X).  out: where to put dX, `dY` or `X` itself included."""
    lib, index, handle, context = _begin(X, stream)
    code, ldx = _code(X, "X"), _ld(X, "X")
    n, d = X.shape
    if dY.shape != X.shape or dY.dtype != X.dtype:
        _refuse("dY has the shape and dtype of X")
    if stats.shape != (n, 2) or stats.dtype != torch.float32 or not stats.is_contiguous():
        _refuse("stats must be the n x 2 float32 tensor of osscar_layernorm_forward")
    _on(index, dY=dY, stats=stats, out=out)
    wp, wc = _gains(index, weight, d, "weight")
    wc = code if wc is None else wc
    if dw_dtype is None:
        dw_dtype = X.dtype if weight is None else weight.dtype
    if dw_dtype not in _CODES:
        _refuse(f"dw_dtype {dw_dtype} is neither float32 nor bfloat16")
    if out is not None and not need_x:
        _refuse("out goes with need_x")
    with context:
        dX = _out(out, X, X.shape) if need_x else None
        dw = db = ws = None
        size, wsp = 0, None
        if need_w:
            dw, db = _EMPTY(d, dtype=dw_dtype, device=X.device), _EMPTY(d, dtype=dw_dtype, device=X.device)
            ws, wsp, size = _workspace(lib.osscar_layernorm_workspace_bytes(n, d), X.device)
        status = lib.osscar_layernorm_backward(X.data_ptr(), n, d, ldx, code, wp, wc, dY.data_ptr(), _ld(dY, "dY"), stats.data_ptr(),
                                               dX.data_ptr() if need_x else None, _ld(dX, "out") if need_x else d, dw.data_ptr() if need_w else None,
                                               db.data_ptr() if need_w else None, _CODES[dw_dtype], wsp, size, handle)
    _done(lib, status)
    return dX, dw, db


def _components(t: torch.Tensor, count: int, rank: int, width: int, what: str) -> Tuple[int, int]:
    """(from one component to the next, from one adapter to the next) of adapters x components x width"""
    after, ld, one = t.stride()
    if one != 1 and width > 1:
        _refuse(f"the components of {what} must be contiguous")
    if rank <= 1:
        ld = width
    if ld < width:
        _refuse(f"the components of {what} overlap")
    return ld or 1, after if count > 1 else 0


def _adapters(X, A, B, index, scale, ranks, at: int):
    """(description, addresses of X, A, B, index, scale, ranks)"""
    code, ldx = _code(X, "X"), _ld(X, "X")
    if A.dtype != X.dtype or B.dtype != X.dtype:
        _refuse("X, A and B have one dtype")
    n, d = X.shape
    if A.dim() != 3 or B.dim() != 3:
        _refuse("A and B are adapters x rank x width")
    (count, rank, width), (b_count, b_rank, m) = A.shape, B.shape
    if width != d or b_count != count or b_rank != rank:
        _refuse("A is adapters x rank x d, B adapters x rank x m")
    if A.get_device() != at or B.get_device() != at:
        _on(at, A=A, B=B)
    lda, next_a = _components(A, count, rank, d, "A")
    ldb, next_b = _components(B, count, rank, m, "B")
    ip = None if index is None else _vector_on(at, index, n, torch.int64, "index")
    sp = None if scale is None else _vector_on(at, scale, count, torch.float32, "scale")
    rp = None if ranks is None else _vector_on(at, ranks, count, torch.int32, "ranks")
    return _AdaptersDesc(n, d, m, ldx, lda, next_a, ldb, next_b, count, rank, code, 0 if index is None else 1), (X.data_ptr(), A.data_ptr(), B.data_ptr(), ip, sp, rp)


def osscar_adapters_forward(X: torch.Tensor, A: torch.Tensor, B: torch.Tensor, index: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                            ranks: Optional[torch.Tensor] = None, base: Optional[torch.Tensor] = None, save: bool = False, out: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None):
    """Row i of Y is base_i + scale_e (X_i A_e^T) B_e with e = index[i]: low-rank adapters beside a projection whose output is `base` (n x m; None: zeros).  X: n x d, A: adapters x rank x d,
    B: adapters x rank x m, one dtype.  index: int64, negative where a row has none; None: all rows have the first.  scale: float32 per adapter.  ranks: int32 per adapter, how
    many of its components count.  out: where to put Y, `base` itself included.  save: returns (Y, T) with the n x rank float32 products X_i A_e^T, else Y."""
    lib, at, handle, context = _begin(X, stream)
    desc, (xp, ap, bp, ip, sp, rp) = _adapters(X, A, B, index, scale, ranks, at)
    n, m = desc.n, desc.m
    if base is not None and (base.shape != (n, m) or base.dtype != X.dtype):
        _refuse("base is n x m, of the dtype of X")
    if base is not None or out is not None:
        _on(at, base=base, out=out)
    with context:
        Y = _out(out, X, (n, m))
        T = _EMPTY(n, desc.rank, dtype=torch.float32, device=X.device) if save else None
        ws, wp, size = _workspace(lib.osscar_adapters_workspace_bytes(C.byref(desc), 0), X.device)
        status = lib.osscar_adapters_forward(C.byref(desc), xp, ap, bp, ip, sp, rp, None if base is None else base.data_ptr(), m if base is None else _ld(base, "base"),
                                             Y.data_ptr(), _ld(Y, "out"), T.data_ptr() if save else None, wp, size, handle)
    _done(lib, status)
    return (Y, T) if save else Y


def osscar_adapters_backward(X: torch.Tensor, A: torch.Tensor, B: torch.Tensor, dY: torch.Tensor, T: Optional[torch.Tensor] = None, index: Optional[torch.Tensor] = None,
                             scale: Optional[torch.Tensor] = None, ranks: Optional[torch.Tensor] = None, base: Optional[torch.Tensor] = None, need_x: bool = True,
                             need_w: bool = True, dw_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """(dX, dA, dB) of osscar_adapters_forward for the gradient dY of Y; None for what is not needed.  T: from forward's save=True (else it is computed again).  base: n x d, what
    dX is added to, as the gradient that came through the projection (None: zeros).  out: where to put dX, `base`, `dY` or `X` itself included.  dw_dtype: float32 or
    bfloat16, by default the adapters'."""
    lib, at, handle, context = _begin(X, stream)
    desc, (xp, ap, bp, ip, sp, rp) = _adapters(X, A, B, index, scale, ranks, at)
    n, d, m, device = desc.n, desc.d, desc.m, X.device
    if dY.shape != (n, m) or dY.dtype != X.dtype:
        _refuse("dY is n x m, of the dtype of X")
    if base is not None and (base.shape != (n, d) or base.dtype != X.dtype):
        _refuse("base is n x d, of the dtype of X")
    if T is not None and (T.shape != (n, desc.rank) or T.dtype != torch.float32 or not T.is_contiguous()):
        _refuse("T must be the n x rank float32 tensor of osscar_adapters_forward")
    if not need_x and (base is not None or out is not None):
        _refuse("base and out go with need_x")
    dw_dtype = X.dtype if dw_dtype is None else dw_dtype
    if dw_dtype not in _CODES:
        _refuse(f"dw_dtype {dw_dtype} is neither float32 nor bfloat16")
    _on(at, dY=dY, T=T, base=base, out=out)
    with context:
        dX = _out(out, X, (n, d)) if need_x else None
        dA = dB = None
        if need_w:
            dA, dB = _EMPTY(A.shape, dtype=dw_dtype, device=device), _EMPTY(B.shape, dtype=dw_dtype, device=device)
        ws, wp, size = _workspace(lib.osscar_adapters_workspace_bytes(C.byref(desc), 1 if need_w else 2), device)
        status = lib.osscar_adapters_backward(C.byref(desc), xp, ap, bp, ip, sp, rp, dY.data_ptr(), _ld(dY, "dY"), None if T is None else T.data_ptr(),
                                              None if base is None else base.data_ptr(), d if base is None else _ld(base, "base"), dX.data_ptr() if need_x else None,
                                              _ld(dX, "out") if need_x else d, dA.data_ptr() if need_w else None, dB.data_ptr() if need_w else None, _CODES[dw_dtype], wp, size,
                                              handle)
    _done(lib, status)
    return dX, dA, dB


_BLOCK = 256


class _StateTensors(NamedTuple):
    m: torch.Tensor
    v: torch.Tensor
    m_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


class AdamWState(_StateTensors):
    """The states of one parameter, in the order of its memory: float32 m and v; or in 8 bits codes of m (float8_e4m3fn) and of sqrt(v) (uint8), with a float32
    scale for every 256 of them.  place: shape and strides of the parameter that 8-bit states were last stepped with."""
    place: Optional[Tuple[Tuple[int, ...], Tuple[int, ...]]] = None


class AdamWValues(NamedTuple):
    """What 8-bit states stand for, in bfloat16 (exactly, but for m of scales below 2^-124, which bfloat16 has fewer bits for): m and the root of v, of the parameter's shape."""
    m: torch.Tensor
    root: torch.Tensor


def _listed(tensors):
    return tensors if tensors is None or type(tensors) is list else list(tensors)


def _rows(params: Optional[list], grads: Optional[list], masters: Optional[list], states: list, bits: int, index: int):
    """The table of osscar_adamw, of tensors as they are now: an address is read at each call, so that none is used after its memory went elsewhere."""
    table = (_AdamWTensor * len(states))()
    why = load_tensors().adamw_rows(C.addressof(table), params, grads, masters, states, bits, index)
    if why is not None:
        _refuse(why)
    return table


def _bits(states: list) -> int:
    first = states[0]
    return 8 if isinstance(first, tuple) and len(first) == 4 and first[2] is not None else 32


def _scalar(t: torch.Tensor, dtype: torch.dtype, what: str, index: int) -> int:
    if t.dtype != dtype or t.numel() != 1 or t.get_device() != index:
        _refuse(f"{what} must be one {dtype} on cuda:{index}")
    return t.data_ptr()


def osscar_adamw(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], states: Sequence[AdamWState], lr: Union[float, torch.Tensor], step: Union[int, torch.Tensor], beta1: float = 0.9,
                 beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01, masters: Optional[Sequence[Optional[torch.Tensor]]] = None, grad_scale: Optional[torch.Tensor] = None,
                 seed: Optional[int] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """One step of AdamW over a list of parameters, in place; autograd does not see it.

    params: float32 or bfloat16 on one GPU, any shape, their elements side by side in memory (a transposed matrix will do).  grads: of the same shapes and layouts, float32 or
    bfloat16.  states: one AdamWState per parameter, all of 32 or all of 8 bits (AdamW(params, bits=8).states makes zeros).  masters: a float32 copy for bfloat16 parameters, or None, as a
    list or None for all.  step counts from 1; lr and step may be tensors of one element on the GPU (float32, int64), which a captured step reads anew at each replay; the tensors of
    the lists it reads and writes where they were when it was captured.  grad_scale: one float32 on the GPU that the gradients are multiplied by; where it is not finite nothing
    changes.  seed (32 bits, another for each step; a step on the GPU is added to it): 8-bit states, and bfloat16 parameters without a master, are rounded up by chance instead of
    to the nearest."""
    params, grads, masters, states = _listed(params), _listed(grads), _listed(masters), _listed(states)
    if not params or not states or len(states) != len(params):
        _refuse("states have one entry per parameter, and there is one parameter at least")
    if grads is None:
        _refuse("no gradients were given")
    lib, index, handle, context = _begin(params[0], stream)
    bits = _bits(states)
    table = _rows(params, grads, masters, states, bits, index)
    desc = _AdamWDesc(0.0, beta1, beta2, eps, weight_decay, 1, None, None, None, 0, 0, bits)
    if isinstance(lr, torch.Tensor):
        desc.lr_dev = _scalar(lr, torch.float32, "lr", index)
    else:
        desc.lr = lr
    if isinstance(step, torch.Tensor):
        desc.step_dev = _scalar(step, torch.int64, "step", index)
    else:
        desc.step = step
    if grad_scale is not None:
        desc.grad_scale_dev = _scalar(grad_scale, torch.float32, "grad_scale", index)
    if seed is not None:
        if not 0 <= seed < 1 << 32:
            _refuse("seed has 32 bits")
        desc.seed, desc.stochastic = seed, 1
    with context:
        status = lib.osscar_adamw(table, len(params), C.byref(desc), handle)
    _done(lib, status)


def osscar_adamw_values(states: Sequence[AdamWState], stream: Optional[torch.cuda.Stream] = None) -> List[AdamWValues]:
    """What 8-bit states stand for, one AdamWValues each, of the shape and layout of the parameter that the state was last stepped with (one that was not: a vector)."""
    states = _listed(states)
    if not states:
        _refuse("no states")
    if _bits(states) != 8:
        _refuse("states of 32 bits are their own values")
    device = states[0][0].device
    lib, index, handle, context = _begin(states[0][0], stream)
    table = _rows(None, None, None, states, 8, index)
    with context:
        values = []
        for row, s in zip(table, states):
            place = getattr(s, "place", None)
            if place is None or math.prod(place[0]) != row.n:
                place = (row.n,), (1,)
            values.append(AdamWValues(*(torch.empty_strided(*place, dtype=torch.bfloat16, device=device) for _ in range(2))))
        outs = C.c_void_p * len(values)
        status = lib.osscar_adamw_values(table, len(values), outs(*(x.m.data_ptr() for x in values)), outs(*(x.root.data_ptr() for x in values)), handle)
    _done(lib, status)
    return values


class AdamW:
    """The lists of osscar_adamw kept together: parameters, masters, states, and the gradients that were given last.

    params, grads, masters: as osscar_adamw takes them; grads may also be given, or given anew, at each step.  states: one AdamWState per parameter, or None: zeros in `bits` bits.  Each step looks
    at the tensors again: one that was moved, as by `p.data = ...`, is stepped where it is now, and one that no longer goes with its state, master or gradient is refused."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Optional[Sequence[torch.Tensor]] = None, bits: Optional[int] = None,
                 masters: Optional[Sequence[Optional[torch.Tensor]]] = None, states: Optional[Sequence[AdamWState]] = None):
        self.params = list(params)
        if not self.params:
            _refuse("no parameters")
        self.masters = [None] * len(self.params) if masters is None else list(masters)
        if states is not None:
            states = [s if isinstance(s, AdamWState) else AdamWState(*s) for s in states]
            if len(states) != len(self.params):
                _refuse("states have one entry per parameter")
        if bits is None:
            bits = 8 if states and states[0].m_scale is not None else 32
        if bits not in (8, 32):
            _refuse("states have 8 or 32 bits")
        self.bits = bits
        index = _begin(self.params[0], None)[1]
        self.states: List[AdamWState] = [self._zeros(p) for p in self.params] if states is None else states
        self.grads: Optional[List[torch.Tensor]] = None if grads is None else list(grads)
        _rows(self.params, self.grads, self.masters, self.states, bits, index)

    def _zeros(self, p: torch.Tensor) -> AdamWState:
        n, device = p.numel(), self.params[0].device
        if self.bits == 32:
            return AdamWState(torch.zeros(n, dtype=torch.float32, device=device), torch.zeros(n, dtype=torch.float32, device=device))
        blocks = -(-n // _BLOCK)
        return AdamWState(torch.zeros(n, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn), torch.zeros(n, dtype=torch.uint8, device=device),
                          torch.zeros(blocks, dtype=torch.float32, device=device), torch.zeros(blocks, dtype=torch.float32, device=device))

    def osscar_adamw(self, lr: Union[float, torch.Tensor], step: Union[int, torch.Tensor], beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01,
                     grads: Optional[Sequence[torch.Tensor]] = None, grad_scale: Optional[torch.Tensor] = None, seed: Optional[int] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> None:
        """osscar_adamw over the lists.  grads: new gradients, kept for later steps."""
        grads = self.grads if grads is None else list(grads)
        osscar_adamw(self.params, grads, self.states, lr, step, beta1, beta2, eps, weight_decay, self.masters, grad_scale, seed, stream)
        self.grads = grads

    def osscar_adamw_values(self, stream: Optional[torch.cuda.Stream] = None) -> List[AdamWValues]:
        """What the 8-bit states stand for, one AdamWValues per parameter, of its shape."""
        index = _begin(self.params[0], None)[1]
        _rows(self.params, None, self.masters, self.states, self.bits, index)      # (a parameter that no longer goes with its state is refused)
        return osscar_adamw_values(self.states, stream)
