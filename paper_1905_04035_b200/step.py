"""Marshalling for the operators of a step around the tied weight (see ``include/dst_step.h`` for the contract):
log probabilities and their gradient, the root-mean-square norm, the gradient norm and clipping.

The functions carry the names of the C entry points.  Matrices are 2-D CUDA tensors with contiguous rows (any distance
between rows); outputs are allocated by the caller.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from .binding import DST_BF16, DST_F32, _Tensor, load_calls, load_library
from .tied import _INDEX, Fp8Matrix, _device, _enqueue, _here, _matrix, _vector, _workspace

DST_LOGPROB_MAX_TOP = 32
DST_RMSNORM_MAX_D = 16384


def _logits(logits: torch.Tensor, targets: Optional[torch.Tensor], other: Optional[torch.Tensor] = None):
    """(device, arguments that every entry for log probabilities starts with, up to the scale, rows, vocab)."""
    index = _device(logits)
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, vocab]")
    rows, vocab = logits.shape
    pl, ld, tl = _matrix(logits, rows, vocab, index, "logits")
    named = targets if targets is not None else other
    index_type = _INDEX.get(torch.int64 if named is None else named.dtype)
    if index_type is None:
        raise TypeError("targets and top_tokens must be int32 or int64, got %s" % named.dtype)
    pt = _vector(targets, rows, None if targets is None else targets.dtype, index, "targets")
    return index, (pl, ld, tl, rows, vocab, pt, index_type), rows, vocab


def _stats(t: Optional[torch.Tensor], rows: int, index: int):
    if t is None:
        return None
    at, n = load_calls().table(t, rows, torch.float32, index, "stats")
    if n != 2:
        raise ValueError("stats must be contiguous [%d, 2]" % rows)
    return at


def _result(t: Optional[torch.Tensor], index: int):
    if t is None:
        return None
    if not t.is_contiguous() or t.numel() * t.element_size() < 24:
        raise ValueError("result must be contiguous and hold 24 bytes")
    _here(t, index)
    return t.data_ptr()


def dst_logprob(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, logprob: Optional[torch.Tensor] = None, *,
                scale: float = 1.0, lse: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None,
                top_tokens: Optional[torch.Tensor] = None, top_logprob: Optional[torch.Tensor] = None,
                result: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue ``dst_logprob``: log probabilities of ``targets`` under softmax(scale * logits), the rows' ``lse`` and
    ``entropy``, ``stats`` [rows, 2] for ``dst_logprob_backward``, and their largest logits as ``top_tokens`` and ``top_logprob`` [rows, n].  Outputs that are not given are
    not computed.  ``result``: an int32/uint8 CUDA tensor of at least 24 bytes that receives ``dst_result_t``."""
    index, head, rows, _ = _logits(logits, targets, top_tokens)
    f32 = torch.float32
    n, tokens, their = 0, None, None
    if top_tokens is not None:
        tokens, n = load_calls().table(top_tokens, rows, torch.int64 if head[6] else torch.int32, index, "top_tokens")
    if top_logprob is not None:
        their, k = load_calls().table(top_logprob, rows, f32, index, "top_logprob")
        if tokens is not None and k != n:
            raise ValueError("top_tokens and top_logprob must have as many columns")
        n = k
    _enqueue("dst_logprob", index, stream, *head, scale, _vector(logprob, rows, f32, index, "logprob"), _vector(lse, rows, f32, index, "lse"),
             _vector(entropy, rows, f32, index, "entropy"), _stats(stats, rows, index), n, tokens, their, _result(result, index))


def dst_logprob_loss(logits: torch.Tensor, targets: Optional[torch.Tensor], dlogprob: Optional[torch.Tensor], logprob: Optional[torch.Tensor],
                     dlogits: torch.Tensor, *, scale: float = 1.0, dentropy: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                     entropy: Optional[torch.Tensor] = None, result: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Enqueue ``dst_logprob_loss``: log probabilities of ``targets`` and, in the same pass, the logits' gradient ``dlogits`` of
    sum(dlogprob * logprob + dentropy * entropy).  ``dlogits`` may be ``logits``."""
    index, head, rows, vocab = _logits(logits, targets)
    f32 = torch.float32
    pd, ldd, td = _matrix(dlogits, rows, vocab, index, "dlogits")
    _enqueue("dst_logprob_loss", index, stream, *head, scale, _vector(dlogprob, rows, f32, index, "dlogprob"), _vector(dentropy, rows, f32, index, "dentropy"),
             _vector(logprob, rows, f32, index, "logprob"), _vector(lse, rows, f32, index, "lse"), _vector(entropy, rows, f32, index, "entropy"),
             pd, ldd, td, _result(result, index))
    return dlogits


def dst_logprob_backward(logits: torch.Tensor, targets: Optional[torch.Tensor], stats: torch.Tensor, dlogprob: Optional[torch.Tensor],
                         dlogits: torch.Tensor, *, scale: float = 1.0, entropy: Optional[torch.Tensor] = None,
                         dentropy: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Enqueue ``dst_logprob_backward``: the gradient of ``dst_logprob_loss`` from ``dst_logprob``'s ``stats`` and, with
    ``dentropy``, ``entropy``.  ``dlogits`` may be ``logits``."""
    index, head, rows, vocab = _logits(logits, targets)
    f32 = torch.float32
    pd, ldd, td = _matrix(dlogits, rows, vocab, index, "dlogits")
    _enqueue("dst_logprob_backward", index, stream, *head, scale, _stats(stats, rows, index), _vector(entropy, rows, f32, index, "entropy"),
             _vector(dlogprob, rows, f32, index, "dlogprob"), _vector(dentropy, rows, f32, index, "dentropy"), pd, ldd, td)
    return dlogits


def dst_rmsnorm(x: torch.Tensor, weight: Optional[torch.Tensor], out: Optional[torch.Tensor] = None, *, q: Optional[Fp8Matrix] = None,
                residual: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None, eps: float = 1e-6,
                inv_rms: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue ``dst_rmsnorm``: the norm of h = x + residual into ``out`` and / or, in 8 bits, into ``q``; h itself into ``sum_out``
    (which may be ``residual``)."""
    index = _device(x)
    if x.dim() != 2:
        raise ValueError("x must be [rows, d]")
    rows, d = x.shape
    px, ldx, tx = _matrix(x, rows, d, index, "x")
    pr = ps = po = None
    ldr = lds = ldo = 0
    ts, to = tx, DST_F32
    if residual is not None:
        pr, ldr, ts = _matrix(residual, rows, d, index, "residual")
    if sum_out is not None:
        ps, lds, t = _matrix(sum_out, rows, d, index, "sum_out")
        if residual is not None and t != ts:
            raise TypeError("residual and sum_out must share a dtype")
        ts = t
    if out is not None:
        po, ldo, to = _matrix(out, rows, d, index, "out")
    if q is not None:
        _here(q.q, index)
    elif out is None:
        raise ValueError("out or q must be given")
    _enqueue("dst_rmsnorm", index, stream, px, ldx, tx, pr, ldr, ps, lds, ts, _vector(weight, d, torch.float32, index, "weight"), eps,
             po, ldo, to, None if q is None else q._c, _vector(inv_rms, rows, torch.float32, index, "inv_rms"), rows, d)


def dst_rmsnorm_backward_workspace_bytes(rows: int, d: int) -> int:
    return int(load_library().dst_rmsnorm_backward_workspace_bytes(rows, d))


def dst_rmsnorm_backward(dy: torch.Tensor, h: torch.Tensor, weight: Optional[torch.Tensor], inv_rms: torch.Tensor, dx: torch.Tensor, *,
                         dsum: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Enqueue ``dst_rmsnorm_backward``: ``dx`` = ``dsum`` + the norm's gradient by h, and ``dweight``.  ``dx`` may be ``dy``, ``h`` or
    ``dsum``."""
    index = _device(dx)
    if dy.dim() != 2:
        raise ValueError("dy must be [rows, d]")
    rows, d = dy.shape
    py, ldy, ty = _matrix(dy, rows, d, index, "dy")
    ph, ldh, th = _matrix(h, rows, d, index, "h")
    px, ldx, tx = _matrix(dx, rows, d, index, "dx")
    ps, lds = None, 0
    if dsum is not None:
        ps, lds, ts = _matrix(dsum, rows, d, index, "dsum")
        if ts != tx:
            raise TypeError("dsum and dx must share a dtype")
    ws, ws_bytes = _workspace(workspace, index)
    f32 = torch.float32
    _enqueue("dst_rmsnorm_backward", index, stream, py, ldy, ty, ph, ldh, th, _vector(weight, d, f32, index, "weight"),
             _vector(inv_rms, rows, f32, index, "inv_rms"), ps, lds, px, ldx, tx, _vector(dweight, d, f32, index, "dweight"), rows, d, ws, ws_bytes)
    return dx


def _apart(spans) -> bool:
    """Whether no two of the (first byte, byte after the last) overlap."""
    spans = sorted(s for s in spans if s[0] < s[1])
    return all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))


class TensorList:
    """A list of contiguous tensors of one CUDA device, fp32 or bf16, laid out for ``dst_grad_norm`` and ``dst_clip``.  It keeps the memory
    alive that the tensors have when the list is made (a tensor that is given other memory later is to be listed anew); the values are read
    when a call runs."""

    def __init__(self, tensors: Sequence[torch.Tensor]):
        self.tensors = [t.detach() for t in tensors]
        self.device_index: Optional[int] = None
        self._c = (_Tensor * max(1, len(self.tensors)))()
        for t, c in zip(self.tensors, self._c):
            index = _device(t)
            if self.device_index is None:
                self.device_index = index
            _here(t, self.device_index)
            if t.dtype not in (torch.float32, torch.bfloat16):
                raise TypeError("tensors must be float32 or bfloat16, got %s" % t.dtype)
            if not t.is_contiguous():
                raise ValueError("tensors must be contiguous")
            c.data, c.n, c.type = t.data_ptr(), t.numel(), DST_F32 if t.dtype == torch.float32 else DST_BF16
        self.distinct = _apart((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in self.tensors)

    def __len__(self) -> int:
        return len(self.tensors)


def _clip(clip: torch.Tensor):
    index = _device(clip)
    return index, _vector(clip, 2, torch.float32, index, "clip")


def _on(tensors: TensorList, index: int) -> None:
    if tensors.device_index is not None and tensors.device_index != index:
        raise ValueError("all tensors must live on the same device")


def dst_grad_norm_workspace_bytes(tensors: TensorList) -> int:
    return int(load_library().dst_grad_norm_workspace_bytes(tensors._c, len(tensors)))


def dst_grad_norm(tensors: TensorList, clip: torch.Tensor, max_norm: float, workspace: Optional[torch.Tensor] = None, *, stream=None) -> torch.Tensor:
    """Enqueue ``dst_grad_norm``: ``clip`` [2] = the norm over all tensors and the factor that brings it down to ``max_norm``."""
    index, pc = _clip(clip)
    _on(tensors, index)
    ws, ws_bytes = _workspace(workspace, index)
    _enqueue("dst_grad_norm", index, stream, tensors._c, len(tensors), max_norm, pc, ws, ws_bytes)
    return clip


def dst_clip(tensors: TensorList, clip: torch.Tensor, outs: Optional[TensorList] = None, *, stream=None) -> None:
    """Enqueue ``dst_clip``: every tensor times ``clip[1]``, into ``outs`` or in place.  An output may be its own tensor; one that shares
    memory with another tensor, or with another output, is refused."""
    index, pc = _clip(clip)
    _on(tensors, index)
    if outs is None:
        outs = tensors
    _on(outs, index)
    if len(outs) != len(tensors):
        raise ValueError("outs must have as many tensors")
    if not outs.distinct:
        raise ValueError("tensors that share memory would be scaled twice")
    _enqueue("dst_clip", index, stream, tensors._c, outs._c, len(tensors), pc)
