"""Marshalling for the operators around the tied weight (see ``include/dst_tied.h`` for the contract).

The functions carry the names of the C entry points; ``Fp8Matrix`` and ``TiedProjection`` own caller-side buffers.
Matrices are 2-D CUDA tensors with contiguous rows (any distance between rows); outputs are allocated by the caller.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from .binding import DST_BF16, DST_F32, DST_I32, DST_I64, DstError, _Dropout, _Fp4, _Fp8, load_calls, load_library

DST_FP8_ROW, DST_FP8_SQUARE = 0, 1
_TYPES = {torch.float32: DST_F32, torch.bfloat16: DST_BF16}
_INDEX = {torch.int32: DST_I32, torch.int64: DST_I64}


# the stream that work goes to unless one is given; torch's own accessor of the raw handle, without a Stream object a call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device   # (a tensor is on a device already)


def _matrix(t: torch.Tensor, rows: int, cols: int, index: int, name: str):
    """(pointer, leading dimension, type) of a [rows, cols] matrix with contiguous rows on CUDA device `index`."""
    return load_calls().matrix(t, rows, cols, index, name)


def _vector(t: Optional[torch.Tensor], n: int, dtype, index: int, name: str):
    """The pointer of n contiguous elements, or None."""
    return None if t is None else load_calls().vector(t, n, dtype, index, name)


def _device(t: torch.Tensor) -> int:
    index = t.get_device()
    if index < 0:
        raise ValueError("tensors must be CUDA tensors")
    return index


def _here(t: torch.Tensor, index: int) -> None:
    if t.get_device() != index:
        raise ValueError("all tensors must live on the same device")


def _enqueue(name: str, index: int, stream, *args) -> None:
    """Call a C entry whose last argument is the stream, with device `index` current; raises on a status."""
    fn = getattr(load_calls(), name)
    if _current_device() == index:
        rc = fn(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(index):
            rc = fn(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    if rc != 0:
        raise DstError(rc, name)


def _drop(p, seed, offset, offset_tensor, row_offset, index) -> _Dropout:
    at = None
    if offset_tensor is not None:
        if offset_tensor.dtype != torch.int64 or offset_tensor.numel() != 1:
            raise TypeError("offset_tensor must hold one int64")
        _here(offset_tensor, index)
        at = offset_tensor.data_ptr()
    return _Dropout(p, seed & 0xFFFFFFFFFFFFFFFF, offset & 0xFFFFFFFFFFFFFFFF, at, row_offset)


def dst_dropout(x: torch.Tensor, out: torch.Tensor, p: float, seed: int, offset: int = 0, *,
                residual: Optional[torch.Tensor] = None, scale: float = 1.0, row_offset: int = 0,
                offset_tensor: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Enqueue ``dst_dropout``: out = residual + scale * dropout(x).  The same call on the output's gradient, without
    the residual, is the gradient of ``x``.  ``out`` may be ``x`` or ``residual``."""
    index = _device(out)
    if x.dim() != 2:
        raise ValueError("x must be [rows, d]")
    rows, d = x.shape
    px, ldx, tx = _matrix(x, rows, d, index, "x")
    po, ldo, to = _matrix(out, rows, d, index, "out")
    pr, ldr = None, 0
    if residual is not None:
        pr, ldr, tr = _matrix(residual, rows, d, index, "residual")
        if tr != to:
            raise TypeError("residual and out must share a dtype")
    drop = _drop(p, seed, offset, offset_tensor, row_offset, index)
    _enqueue("dst_dropout", index, stream, px, ldx, tx, pr, ldr, po, ldo, to, rows, d, scale, drop)
    return out


def dst_embed(indices: torch.Tensor, weight: torch.Tensor, out: torch.Tensor, *, scale: float = 1.0,
              position: Optional[torch.Tensor] = None, p: float = 0.0, seed: int = 0, offset: int = 0,
              row_offset: int = 0, offset_tensor: Optional[torch.Tensor] = None, result: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """Enqueue ``dst_embed``: out = dropout(scale * weight[indices] + position rows).  Its gradient's value rows are
    ``dst_dropout(grad, values, p, seed, offset, scale=scale)``, which ``dst_densify`` takes with ``indices``.

    ``result``: an int32/uint8 CUDA tensor of at least 24 bytes that receives ``dst_result_t``."""
    index_type = _INDEX.get(indices.dtype)
    if index_type is None:
        raise TypeError("indices must be int32 or int64, got %s" % indices.dtype)
    index = _device(out)
    if indices.dim() != 1 or weight.dim() != 2:
        raise ValueError("indices must be 1-D and weight [vocab, d]")
    n, (vocab, d) = indices.shape[0], weight.shape
    pi = _vector(indices, n, indices.dtype, index, "indices")
    pw, ldw, tw = _matrix(weight, vocab, d, index, "weight")
    po, ldo, to = _matrix(out, n, d, index, "out")
    if (ldw != d and vocab > 1) or (ldo != d and n > 1):
        raise ValueError("weight and out must be contiguous")
    n_pos, pp = 0, None
    if position is not None:
        n_pos = position.shape[0] if position.dim() == 2 else 0
        pp, ldp, tp = _matrix(position, n_pos, d, index, "position")
        if tp != DST_F32:
            raise TypeError("position must be float32, got %s" % position.dtype)
        if ldp != d and n_pos > 1:
            raise ValueError("position must be contiguous [n_positions, d]")
    pres = None
    if result is not None:
        if not result.is_contiguous() or result.numel() * result.element_size() < 24:
            raise ValueError("result must be contiguous and hold 24 bytes")
        _here(result, index)
        pres = result.data_ptr()
    drop = _drop(p, seed, offset, offset_tensor, row_offset, index)
    _enqueue("dst_embed", index, stream, pi, n, index_type, pw, vocab, d, tw, pp, n_pos, po, to, scale, drop, pres)
    return out


class Fp8Matrix:
    """Owns a matrix [rows, cols] in 8-bit floating point (``dst_fp8_t``): ``q`` [rows, cols padded to 16] and a scale
    (a power of two, as its exponent + 127) for each block of 128 columns of a row (``DST_FP8_ROW``) or 128 x 128
    (``DST_FP8_SQUARE``), in ``scale`` [rows / 128, column blocks / 4, 512]."""

    def __init__(self, rows: int, cols: int, block: int = DST_FP8_ROW, *, device="cuda"):
        if block not in (DST_FP8_ROW, DST_FP8_SQUARE):
            raise ValueError("block must be DST_FP8_ROW or DST_FP8_SQUARE")
        if rows < 0 or cols < 0:
            raise ValueError("rows and cols must not be negative")
        self.rows, self.cols, self.block = rows, cols, block
        self.q = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.float8_e4m3fn, device=device)
        self.scale = torch.empty(-(-rows // 128), -(-cols // 512), 512, dtype=torch.uint8, device=device)
        self.device = self.q.device
        self._c = _Fp8(self.q.data_ptr(), self.scale.data_ptr(), rows, cols, self.q.shape[1], self.scale.shape[1], block, 0)

    def part(self, rows: int, cols: int) -> "Fp8Matrix":
        """The same buffers seen as a smaller matrix (leading dimensions stay)."""
        if not (0 <= rows <= self.rows and 0 <= cols <= self.cols):
            raise ValueError("a part is at most [%d, %d]" % (self.rows, self.cols))
        m = object.__new__(Fp8Matrix)
        m.rows, m.cols, m.block, m.q, m.scale, m.device = rows, cols, self.block, self.q[:rows], self.scale, self.device
        m._c = _Fp8(self._c.q, self._c.scale, rows, cols, self._c.ld, self._c.ld_scale, self.block, 0)
        return m

    def scales(self) -> torch.Tensor:
        """The scale of every row and column block, fp32 [rows, column blocks]."""
        tiles, groups = self.scale.shape[:2]
        e = self.scale.view(tiles, groups, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(tiles * 128, groups * 4)
        e = e[:self.rows, :-(-self.cols // 128)].int()
        return torch.where(e == 255, torch.nan, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e - 127))

    def dequantize(self) -> torch.Tensor:
        """The fp32 matrix that the 8-bit one stands for."""
        return self.q[:, :self.cols].float() * self.scales().repeat_interleave(128, 1)[:, :self.cols]


class Fp4Matrix:
    """Owns a matrix [rows, cols] in 4-bit floating point (``dst_fp4_t``): ``q`` [rows, bytes padded to 16], two columns a byte, and a
    scale (a power of two, as its exponent + 127) for each block of 32 columns of a row, in ``scale`` [rows / 128, blocks / 4, 512]."""

    def __init__(self, rows: int, cols: int, *, device="cuda"):
        if rows < 0 or cols < 0:
            raise ValueError("rows and cols must not be negative")
        self.rows, self.cols = rows, cols
        self.q = torch.empty(rows, -(-cols // 32) * 16, dtype=torch.uint8, device=device)
        self.scale = torch.empty(-(-rows // 128), -(-cols // 128), 512, dtype=torch.uint8, device=device)
        self.device = self.q.device
        self._c = _Fp4(self.q.data_ptr(), self.scale.data_ptr(), rows, cols, self.q.shape[1], self.scale.shape[1])

    def part(self, rows: int, cols: int) -> "Fp4Matrix":
        """The same buffers seen as a smaller matrix (leading dimensions stay), to be quantised into.  Of what they hold already it is the
        first rows and columns where ``cols`` is a multiple of 128 or all there are: a product reads up to such a multiple."""
        if not (0 <= rows <= self.rows and 0 <= cols <= self.cols):
            raise ValueError("a part is at most [%d, %d]" % (self.rows, self.cols))
        m = object.__new__(Fp4Matrix)
        m.rows, m.cols, m.q, m.scale, m.device = rows, cols, self.q[:rows], self.scale, self.device
        m._c = _Fp4(self._c.q, self._c.scale, rows, cols, self._c.ld, self._c.ld_scale)
        return m

    def scales(self) -> torch.Tensor:
        """The scale of every row and block, fp32 [rows, blocks]."""
        tiles, groups = self.scale.shape[:2]
        e = self.scale.view(tiles, groups, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(tiles * 128, groups * 4)
        e = e[:self.rows, :-(-self.cols // 32)].int()
        return torch.where(e == 255, torch.nan, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e - 127))

    def codes(self) -> torch.Tensor:
        """The elements before scaling, fp32 [rows, cols]."""
        value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=self.device)
        return value[torch.stack([self.q & 15, self.q >> 4], -1).reshape(self.rows, -1)[:, :self.cols].long()]

    def dequantize(self) -> torch.Tensor:
        """The fp32 matrix that the 4-bit one stands for."""
        return self.codes() * self.scales().repeat_interleave(32, 1)[:, :self.cols]


def dst_quantize_fp8(x: torch.Tensor, q: Optional[Fp8Matrix], qt: Optional[Fp8Matrix] = None, *, stream=None) -> None:
    """Enqueue ``dst_quantize_fp8``: x into ``q`` and its transpose into ``qt`` (either may be None)."""
    if q is None and qt is None:
        raise ValueError("q or qt must be given")
    index = _device(x)
    if x.dim() != 2:
        raise ValueError("x must be [rows, cols]")
    rows, cols = x.shape
    px, ldx, tx = _matrix(x, rows, cols, index, "x")
    for m in (q, qt):
        if m is not None:
            _here(m.q, index)
    _enqueue("dst_quantize_fp8", index, stream, px, ldx, tx, rows, cols, None if q is None else q._c, None if qt is None else qt._c)


def dst_matmul_fp8_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load_library().dst_matmul_fp8_workspace_bytes(M, N, K))


def dst_linear_fp8_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load_library().dst_linear_fp8_workspace_bytes(M, N, K))


def _workspace(t: Optional[torch.Tensor], index: int):
    if t is None:
        return None, 0
    _here(t, index)
    if not t.is_contiguous():                               # (of an expanded tensor there is less than its elements say)
        raise ValueError("workspace must be contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def dst_matmul_fp8(a: Fp8Matrix, b: Fp8Matrix, out: torch.Tensor, workspace: Optional[torch.Tensor] = None, *,
                   stream=None) -> torch.Tensor:
    """Enqueue ``dst_matmul_fp8``: out [a.rows, b.rows] = a b^T."""
    index = _device(out)
    _here(a.q, index)
    _here(b.q, index)
    po, ldo, to = _matrix(out, a.rows, b.rows, index, "out")
    ws, ws_bytes = _workspace(workspace, index)
    _enqueue("dst_matmul_fp8", index, stream, a._c, b._c, po, ldo, to, ws, ws_bytes)
    return out


def dst_linear_fp8(x: torch.Tensor, w: Fp8Matrix, out: torch.Tensor, workspace: Optional[torch.Tensor] = None, *,
                   stream=None) -> torch.Tensor:
    """Enqueue ``dst_linear_fp8``: out [x.rows, w.rows] = quantised(x) w^T."""
    index = _device(out)
    if x.dim() != 2:
        raise ValueError("x must be [rows, cols]")
    m = x.shape[0]
    px, ldx, tx = _matrix(x, m, w.cols, index, "x")
    po, ldo, to = _matrix(out, m, w.rows, index, "out")
    _here(w.q, index)
    ws, ws_bytes = _workspace(workspace, index)
    _enqueue("dst_linear_fp8", index, stream, px, ldx, tx, m, w._c, po, ldo, to, ws, ws_bytes)
    return out


def dst_quantize_fp4(x: torch.Tensor, q: Fp4Matrix, *, stream=None) -> None:
    """Enqueue ``dst_quantize_fp4``: x into ``q``."""
    index = _device(x)
    if x.dim() != 2:
        raise ValueError("x must be [rows, cols]")
    rows, cols = x.shape
    px, ldx, tx = _matrix(x, rows, cols, index, "x")
    _here(q.q, index)
    _enqueue("dst_quantize_fp4", index, stream, px, ldx, tx, rows, cols, q._c)


def dst_matmul_fp4_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load_library().dst_matmul_fp4_workspace_bytes(M, N, K))


def dst_linear_fp4_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load_library().dst_linear_fp4_workspace_bytes(M, N, K))


def dst_matmul_fp4(a: Fp4Matrix, b: Fp4Matrix, out: torch.Tensor, workspace: Optional[torch.Tensor] = None, *,
                   stream=None) -> torch.Tensor:
    """Enqueue ``dst_matmul_fp4``: out [a.rows, b.rows] = a b^T."""
    index = _device(out)
    _here(a.q, index)
    _here(b.q, index)
    po, ldo, to = _matrix(out, a.rows, b.rows, index, "out")
    ws, ws_bytes = _workspace(workspace, index)
    _enqueue("dst_matmul_fp4", index, stream, a._c, b._c, po, ldo, to, ws, ws_bytes)
    return out


def dst_linear_fp4(x: torch.Tensor, w: Fp4Matrix, out: torch.Tensor, workspace: Optional[torch.Tensor] = None, *,
                   stream=None) -> torch.Tensor:
    """Enqueue ``dst_linear_fp4``: out [x.rows, w.rows] = quantised(x) w^T."""
    index = _device(out)
    if x.dim() != 2:
        raise ValueError("x must be [rows, cols]")
    m = x.shape[0]
    px, ldx, tx = _matrix(x, m, w.cols, index, "x")
    po, ldo, to = _matrix(out, m, w.rows, index, "out")
    _here(w.q, index)
    ws, ws_bytes = _workspace(workspace, index)
    _enqueue("dst_linear_fp4", index, stream, px, ldx, tx, m, w._c, po, ldo, to, ws, ws_bytes)
    return out


def dst_sample(logits: torch.Tensor, uniform: torch.Tensor, tokens: torch.Tensor, *,
               temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
               top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None,
               prob: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Enqueue ``dst_sample``: a token per row of ``logits`` from the row's uniform number and filters."""
    token_type = _INDEX.get(tokens.dtype)
    if token_type is None:
        raise TypeError("tokens must be int32 or int64, got %s" % tokens.dtype)
    index = _device(logits)
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, vocab]")
    rows, vocab = logits.shape
    pl, ld, tl = _matrix(logits, rows, vocab, index, "logits")
    f32 = torch.float32
    pu = _vector(uniform, rows, f32, index, "uniform")
    pt = _vector(temperature, rows, f32, index, "temperature")
    pk = _vector(top_k, rows, torch.int32, index, "top_k")
    pp = _vector(top_p, rows, f32, index, "top_p")
    pm = _vector(min_p, rows, f32, index, "min_p")
    po = _vector(tokens, rows, tokens.dtype, index, "tokens")
    pb = _vector(prob, rows, f32, index, "prob")
    _enqueue("dst_sample", index, stream, pl, ld, tl, rows, vocab, pu, pt, pk, pp, pm, po, token_type, pb)
    return tokens


class TiedProjection:
    """The pre-softmax projection through the tied weight [vocab, d] in 8-bit floating point, for up to ``max_tokens``
    rows a call: owns the quantised weight and the workspaces, the arithmetic stays in the library.

    With ``bits=4`` the weight and the rows are in 4 bits instead, half the bytes, for answers and scoring (``training=False``): there is
    no gradient through it.

    ``update(weight)`` quantises the weight (after every optimizer step), ``logits(x, out)`` is x W^T, and with
    ``training`` ``backward(dlogits, x, dx, dweight)`` gives both gradients; ``dweight`` is the dense partner that
    ``dst_densify`` adds to the embedding's gradient.

    The calls of one object share its workspace and its quantised weight and gradients: they must be ordered among each other, by
    going to one stream or by events between streams.  Calls that may overlap on the GPU take an object each."""

    def __init__(self, vocab: int, d: int, max_tokens: int, *, training: bool = True, bits: int = 8, device="cuda"):
        if bits not in (4, 8):
            raise ValueError("bits must be 8 or 4")
        if bits == 4 and training:
            raise ValueError("a projection in 4 bits has no gradient: training=False")
        self.vocab, self.d, self.max_tokens, self.training, self.bits = vocab, d, max_tokens, training, bits
        self.weight = Fp4Matrix(vocab, d, device=device) if bits == 4 else Fp8Matrix(vocab, d, DST_FP8_SQUARE, device=device)
        self.device = self.weight.device
        need = (dst_linear_fp4_workspace_bytes if bits == 4 else dst_linear_fp8_workspace_bytes)(max_tokens, vocab, d)
        if training:
            # everything backward needs is there from the start: nothing is allocated, or freed, under a caller's stream
            self.weight_t = Fp8Matrix(d, vocab, DST_FP8_SQUARE, device=device)
            self.grad = Fp8Matrix(max_tokens, vocab, device=device)
            self.grad_t = Fp8Matrix(vocab, max_tokens, device=device)
            self.x_t = Fp8Matrix(d, max_tokens, device=device)
            need = max(need, dst_matmul_fp8_workspace_bytes(max_tokens, d, vocab),
                       dst_matmul_fp8_workspace_bytes(vocab, d, max_tokens))
        self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)

    def update(self, weight: torch.Tensor, stream=None) -> None:
        if self.bits == 4:
            return dst_quantize_fp4(weight, self.weight, stream=stream)
        dst_quantize_fp8(weight, self.weight, self.weight_t if self.training else None, stream=stream)

    def _check(self, tokens: int) -> None:
        if tokens > self.max_tokens:
            raise ValueError("at most %d tokens a call, got %d" % (self.max_tokens, tokens))

    def logits(self, x, out: torch.Tensor, stream=None) -> torch.Tensor:
        """out [tokens, vocab] = x W^T; x is a tensor [tokens, d] or already quantised: an ``Fp8Matrix``, as ``dst_rmsnorm`` writes it, or
        with ``bits=4`` an ``Fp4Matrix``."""
        if isinstance(x, (Fp8Matrix, Fp4Matrix)):
            if isinstance(x, Fp4Matrix) != (self.bits == 4):
                raise TypeError("x must be quantised as the weight is, to %d bits" % self.bits)
            self._check(x.rows)
            return (dst_matmul_fp4 if self.bits == 4 else dst_matmul_fp8)(x, self.weight, out, self.workspace, stream=stream)
        self._check(x.shape[0])
        if self.bits == 4:
            return dst_linear_fp4(x, self.weight, out, self.workspace, stream=stream)
        return dst_linear_fp8(x, self.weight, out, self.workspace, stream=stream)

    def backward(self, dlogits: torch.Tensor, x: torch.Tensor, dx: torch.Tensor, dweight: torch.Tensor, stream=None) -> None:
        """dx [tokens, d] = dlogits W and dweight [vocab, d] = dlogits^T x."""
        if not self.training:
            raise ValueError("the projection was made without training=True")
        m = x.shape[0]
        self._check(m)
        g, gt, xt = self.grad.part(m, self.vocab), self.grad_t.part(self.vocab, m), self.x_t.part(self.d, m)
        dst_quantize_fp8(dlogits, g, gt, stream=stream)
        dst_quantize_fp8(x, None, xt, stream=stream)
        dst_matmul_fp8(g, self.weight_t, dx, self.workspace, stream=stream)
        dst_matmul_fp8(gt, xt, dweight, self.workspace, stream=stream)
