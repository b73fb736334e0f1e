"""Training-step operators next to the optimizer (the second half of
``include/lionmuon.h``): token log probabilities with entropy, top alternatives
and gradient, from logits or from hidden states without them; RMS norm with the
residual's addition, an 8-bit output and gradient; 8-bit activation checkpoints,
8-bit weights and the linear layer's products with them (forward, input
gradient, weight gradient); the norm of queries and keys with their rotation by
position, and its gradient.

Argument marshalling only: results and workspaces are torch tensors, allocated
on the stream that the call runs on.  Matrices are torch tensors whose last
dimension has stride 1 and whose other dimensions fold into rows of one pitch;
anything else raises ValueError (the library copies nothing behind the
caller's back).  Tensors that come from another stream than the call's follow
torch's usual rules: order the streams, and ``record_stream`` what may be
freed early.
"""

from __future__ import annotations

import math
import struct
from typing import NamedTuple, Optional

import torch

from . import lionmuon as _L
from .lionmuon import LM_BF16, LM_F32, LmCheckpoint8, LmMatrix, LmTensor, LmTokenLogprobArgs

GROUP = 128                                   # channels that share one scale (LM_CODE_GROUP)
FORMATS = {"i8": 0, "e4m3": 1}                # lm_code_format
_DTYPES = {torch.float32: LM_F32, torch.bfloat16: LM_BF16}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _dtype(t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _matrix_fields(t, what: str):
    """lm_matrix's fields of a tensor (a vector is one row)."""
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what}: unsupported dtype {t.dtype}")
    dims = t.dim()
    if dims != 2:
        if dims == 0:
            raise ValueError(f"{what}: a scalar is no matrix")
        if dims == 1:
            t = t.unsqueeze(0)
        else:
            try:   # (the rows spelt out: -1 says nothing where there are no elements)
                t = t.view(math.prod(t.shape[:-1]), t.shape[-1])
            except RuntimeError:
                raise ValueError(f"{what}: the leading dimensions do not fold into rows of one pitch") from None
    rows, cols = t.shape
    ld, one = t.stride()
    if one != 1 and cols > 1 and rows > 0:
        raise ValueError(f"{what}: the last dimension must have stride 1")
    return t.data_ptr(), rows, cols, ld if rows > 1 else cols, code


def _matrix(t, what: str) -> LmMatrix:
    return LmMatrix(*_matrix_fields(t, what))


# Structs as their bytes, field by field: cheaper to make than ctypes objects.
_MATRIX = "QqqqI4x"
_NO_MATRIX = (0, 0, 0, 0, 0)
_pack_matrix = struct.Struct("=" + _MATRIX).pack
_pack_checkpoint8 = struct.Struct("=QQqqqqI4x").pack
_pack_weight8 = struct.Struct("=QQqqqq").pack
_pack_linear_logprob = struct.Struct("=" + 2 * _MATRIX + "7Q" + 2 * _MATRIX + "i4x").pack
_HEADS, _TENSOR = "Qqqqqqi4x", "Qqqi4x"
_NO_HEADS, _NO_TENSOR = (0,) * 7, (0,) * 4
_NO_PART = 3 * _NO_HEADS + 2 * _NO_TENSOR
_pack_qk_rotary = struct.Struct("=" + 2 * (3 * _HEADS + 2 * _TENSOR) + "QQqiii4xd").pack


def _vector_fields(t, what: str):
    if t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous vector")
    return t.data_ptr(), 1, t.shape[0], _dtype(t)


def _vector(t, what: str) -> LmTensor:
    return LmTensor(*_vector_fields(t, what))


def _array(t, n: int, dtype, what: str):
    """Address of a dense array of n elements, None for None."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{what}: expected {dtype}, got {t.dtype}")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what}: expected {n} contiguous elements")
    return t.data_ptr()


def _stream_of(t) -> int:
    """The current stream of t's device.  (A call with stream= runs under
    torch.cuda.stream(stream): its new tensors belong to that stream.)"""
    index = t.device.index
    if index is not None and _raw_stream is not None:
        return _raw_stream(index)
    return torch.cuda.current_stream().cuda_stream


class Checkpoint8:
    """An 8-bit checkpoint (``lm_checkpoint8``): ``codes``, uint8, rows x pitch
    with the pitch a multiple of 16; ``scales``, float32, groups of 128 channels
    x (at least) rows, powers of two as ``checkpoint8`` writes them; ``cols``
    channels; ``format`` "i8" or "e4m3"."""

    __slots__ = ("codes", "scales", "cols", "format")

    def __init__(self, codes, scales, cols: int, format: str):
        if format not in FORMATS:
            raise ValueError(f"format {format!r} is not one of {sorted(FORMATS)}")
        if codes.dtype != torch.uint8 or scales.dtype != torch.float32:
            raise TypeError("codes are uint8 and scales float32")
        if codes.dim() != 2 or codes.stride(1) != 1 or codes.shape[1] < cols:
            raise ValueError("codes: expected rows x at least cols bytes, the last dimension of stride 1")
        if scales.dim() != 2 or scales.shape[0] != -(-cols // GROUP) or scales.shape[1] < codes.shape[0] or \
                (scales.shape[1] > 1 and scales.stride(1) != 1):
            raise ValueError("scales: expected groups x at least rows, the last dimension of stride 1")
        self.codes, self.scales, self.cols, self.format = codes, scales, int(cols), format

    @classmethod
    def empty(cls, rows: int, cols: int, format: str, device="cuda") -> "Checkpoint8":
        if format not in FORMATS:
            raise ValueError(f"format {format!r} is not one of {sorted(FORMATS)}")
        c = cls.__new__(cls)
        c.codes = torch.empty((rows, -(-cols // 16) * 16), dtype=torch.uint8, device=device)
        c.scales = torch.empty((-(-cols // GROUP), rows), dtype=torch.float32, device=device)
        c.cols, c.format = cols, format
        return c

    @property
    def rows(self) -> int:
        return self.codes.shape[0]

    def nbytes(self) -> int:
        return self.codes.numel() + 4 * self.scales.numel()

    def fields(self):
        """lm_checkpoint8's."""
        codes, scales = self.codes, self.scales
        rows, pitch = codes.shape
        groups, lds = scales.shape
        # (one row of a wider buffer keeps its buffer's pitch, as several do)
        return (codes.data_ptr(), scales.data_ptr(), rows, self.cols, codes.stride(0) if rows > 1 else max(codes.stride(0), pitch),
                scales.stride(0) if groups > 1 else lds, FORMATS[self.format])

    def desc(self) -> LmCheckpoint8:
        return LmCheckpoint8(*self.fields())

    def unpack(self, dtype=torch.bfloat16, out=None, stream=None):
        """The values the checkpoint stands for (exact in bf16 and in fp32)."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.unpack(dtype, out)
        lib = _L.load_library()
        codes = self.codes
        if out is None:
            out = torch.empty((codes.shape[0], self.cols), dtype=dtype, device=codes.device)
        st = lib.lm_checkpoint8_unpack(self.desc(), _matrix(out, "out"), _stream_of(codes))
        if st:
            _L._check(lib, st, "lm_checkpoint8_unpack")
        return out


def checkpoint8(x, format: str = "e4m3", out: Optional[Checkpoint8] = None, stream=None) -> Checkpoint8:
    """Keep x (bf16 or fp32; leading dimensions fold into rows) in 8 bits."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return checkpoint8(x, format, out)
    lib = _L.load_library()
    m = _matrix(x, "x")
    if out is None:
        out = Checkpoint8.empty(m.rows, m.cols, format, x.device)
    st = lib.lm_checkpoint8_pack(m, out.desc(), _stream_of(x))
    if st:
        _L._check(lib, st, "lm_checkpoint8_pack")
    return out


def linear_wgrad8(dy, x: Checkpoint8, out=None, accumulate: bool = False, dtype=torch.bfloat16, stream=None):
    """dy^T x, the weight gradient (out x in) of y = x W^T whose input was kept
    in 8 bits; ``out`` receives it, or has it added with ``accumulate``."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return linear_wgrad8(dy, x, out, accumulate, dtype)
    lib = _L.load_library()
    if accumulate and out is None:
        raise ValueError("accumulate adds to out: give it")
    m, c = _matrix(dy, "dy"), x.desc()
    if out is None:
        out = torch.empty((m.cols, x.cols), dtype=dtype, device=dy.device)
    w = _matrix(out, "out")
    need = lib.lm_linear_wgrad8_workspace(m, c, w)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    st = lib.lm_linear_wgrad8(m, c, w, 1 if accumulate else 0, ws.data_ptr() if need else None, need, _stream_of(dy))
    if st:
        _L._check(lib, st, "lm_linear_wgrad8")
    return out


class Weight8:
    """8-bit weights of a linear layer (``lm_weight8``): ``codes``, uint8 (e4m3),
    out x pitch with the pitch a multiple of 16; ``scales``, float32, one for each
    block of 128 x 128, powers of two as ``weight8`` writes them (``linear8`` and
    ``linear8_grad`` take any other for NaN, 0 for 2^-127); ``cols`` input channels."""

    __slots__ = ("codes", "scales", "cols")

    def __init__(self, codes, scales, cols: int):
        if codes.dtype != torch.uint8 or scales.dtype != torch.float32:
            raise TypeError("codes are uint8 and scales float32")
        if codes.dim() != 2 or codes.stride(1) != 1 or codes.shape[1] < cols:
            raise ValueError("codes: expected rows x at least cols bytes, the last dimension of stride 1")
        if scales.dim() != 2 or scales.shape[0] != -(-codes.shape[0] // GROUP) or scales.shape[1] < -(-cols // GROUP) or \
                (scales.shape[1] > 1 and scales.stride(1) != 1):
            raise ValueError("scales: expected blocks of rows x at least blocks of columns, the last dimension of stride 1")
        self.codes, self.scales, self.cols = codes, scales, int(cols)

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "Weight8":
        w = cls.__new__(cls)
        w.codes = torch.empty((rows, -(-cols // 16) * 16), dtype=torch.uint8, device=device)
        w.scales = torch.empty((-(-rows // GROUP), -(-cols // GROUP)), dtype=torch.float32, device=device)
        w.cols = cols
        return w

    @property
    def rows(self) -> int:
        return self.codes.shape[0]

    def nbytes(self) -> int:
        return self.codes.numel() + 4 * self.scales.numel()

    def fields(self):
        """lm_weight8's."""
        codes, scales = self.codes, self.scales
        rows, pitch = codes.shape
        down, across = scales.shape
        return (codes.data_ptr(), scales.data_ptr(), rows, self.cols, codes.stride(0) if rows > 1 else max(codes.stride(0), pitch),
                scales.stride(0) if down > 1 else across)

    def unpack(self, dtype=torch.bfloat16, out=None, stream=None):
        """The values the codes stand for (exact in bf16 and in fp32)."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.unpack(dtype, out)
        lib = _L.load_library()
        codes = self.codes
        if out is None:
            out = torch.empty((codes.shape[0], self.cols), dtype=dtype, device=codes.device)
        st = lib.lm_weight8_unpack(_pack_weight8(*self.fields()), _pack_matrix(*_matrix_fields(out, "out")), _stream_of(codes))
        if st:
            _L._check(lib, st, "lm_weight8_unpack")
        return out


def weight8(w, out: Optional[Weight8] = None, stream=None) -> Weight8:
    """Weights (out x in, bf16 or fp32) in 8 bits."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return weight8(w, out)
    lib = _L.load_library()
    m = _matrix_fields(w, "w")
    if out is None:
        out = Weight8.empty(m[1], m[2], w.device)
    st = lib.lm_weight8_pack(_pack_matrix(*m), _pack_weight8(*out.fields()), _stream_of(w))
    if st:
        _L._check(lib, st, "lm_weight8_pack")
    return out


def _linear8(fn: str, x: Checkpoint8, w: Weight8, cols: int, out, dtype, grad: int):
    lib = _L.load_library()
    cx, cw = _pack_checkpoint8(*x.fields()), _pack_weight8(*w.fields())
    if out is None:
        out = torch.empty((x.codes.shape[0], cols), dtype=dtype, device=x.codes.device)
    m = _pack_matrix(*_matrix_fields(out, "out"))
    need = lib.lm_linear8_workspace(cx, cw, grad)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    st = getattr(lib, fn)(cx, cw, m, ws.data_ptr() if need else None, need, _stream_of(x.codes))
    if st:
        _L._check(lib, st, fn)
    return out


def linear8(x: Checkpoint8, w: Weight8, out=None, dtype=torch.bfloat16, stream=None):
    """x W^T: the forward product of a linear layer whose input (e4m3) and
    weights are kept in 8 bits."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return linear8(x, w, out, dtype)
    return _linear8("lm_linear8", x, w, w.rows, out, dtype, 0)


def linear8_grad(dy: Checkpoint8, w: Weight8, out=None, dtype=torch.bfloat16, stream=None):
    """dy W: the input gradient of the same layer, dy in 8 bits (e4m3).  (The
    weight gradient is ``linear_wgrad8``.)"""
    if stream is not None:
        with torch.cuda.stream(stream):
            return linear8_grad(dy, w, out, dtype)
    return _linear8("lm_linear8_grad", dy, w, w.cols, out, dtype, 1)


class RmsNorm(NamedTuple):
    """``y``; ``h`` = x + residual (x itself without one); ``rstd``, one a row;
    ``checkpoint``: y in 8 bits, or None."""
    y: Optional[torch.Tensor]
    h: torch.Tensor
    rstd: torch.Tensor
    checkpoint: Optional[Checkpoint8]


def rmsnorm(x, weight=None, residual=None, eps: float = 1e-6, checkpoint: Optional[str] = None, y: bool = True,
            stream=None) -> RmsNorm:
    """RMS norm of x (+ residual).  ``checkpoint``: the format of an 8-bit copy
    of the output; ``y=False`` leaves the 16- or 32-bit output out."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return rmsnorm(x, weight, residual, eps, checkpoint, y)
    lib = _L.load_library()
    mx = _matrix(x, "x")
    shape = x.shape
    out = x.new_empty(shape) if y else None
    rstd = torch.empty(shape[:-1], dtype=torch.float32, device=x.device)
    kept = Checkpoint8.empty(mx.rows, mx.cols, checkpoint, x.device) if checkpoint is not None else None
    h, mr, mh = x, None, None
    if residual is not None:
        h = x.new_empty(shape)
        mr, mh = _matrix(residual, "residual"), _matrix(h, "h")
    st = lib.lm_rmsnorm(mx, mr, _vector(weight, "weight") if weight is not None else None, eps, mh,
                        _matrix(out, "y") if y else None, rstd.data_ptr(), kept.desc() if kept is not None else None,
                        _stream_of(x))
    if st:
        _L._check(lib, st, "lm_rmsnorm")
    return RmsNorm(out, h, rstd, kept)


def rmsnorm_grad(dy, h, rstd, weight=None, dh=None, dx=None, dweight: bool = True, stream=None):
    """(dx, dweight) of ``rmsnorm``.  ``h``: the stored h, or its Checkpoint8;
    ``dh``: the gradient that reaches h past the norm (the residual stream's);
    ``dx``: the tensor that receives the gradient of x and of residual alike
    (dy or dh themselves are allowed).  dweight has the dtype of weight."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return rmsnorm_grad(dy, h, rstd, weight, dh, dx, dweight)
    lib = _L.load_library()
    m = _matrix(dy, "dy")
    if dx is None:
        dx = dy.new_empty(dy.shape)
    dw = ws = None
    need = 0
    if dweight:
        dw = torch.empty(m.cols, dtype=weight.dtype if weight is not None else torch.float32, device=dy.device)
        need = lib.lm_rmsnorm_grad_workspace(m.rows, m.cols)
        if need:
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    kept = isinstance(h, Checkpoint8)
    st = lib.lm_rmsnorm_grad(m, None if kept else _matrix(h, "h"), h.desc() if kept else None,
                             _array(rstd, m.rows, torch.float32, "rstd"),
                             _vector(weight, "weight") if weight is not None else None,
                             _matrix(dh, "dh") if dh is not None else None, _matrix(dx, "dx"),
                             _vector(dw, "dweight") if dweight else None, ws.data_ptr() if need else None, need,
                             _stream_of(dy))
    if st:
        _L._check(lib, st, "lm_rmsnorm_grad")
    return dx, dw


class TokenLogprob(NamedTuple):
    """One entry a row; ``top_logp`` and ``top_index`` rows x top_k or None;
    ``logp`` None without targets; ``dlogits`` None without weights."""
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    lse: torch.Tensor
    top_logp: Optional[torch.Tensor]
    top_index: Optional[torch.Tensor]
    dlogits: Optional[torch.Tensor]


def _logprob_args(logits, targets, g_logp, g_entropy, g_lse, dlogits):
    m = _matrix(logits, "logits")
    a = LmTokenLogprobArgs()
    a.logits = m
    a.targets = _array(targets, m.rows, torch.int64, "targets")
    a.g_logp = _array(g_logp, m.rows, torch.float32, "g_logp")
    a.g_entropy = _array(g_entropy, m.rows, torch.float32, "g_entropy")
    a.g_lse = _array(g_lse, m.rows, torch.float32, "g_lse")
    if dlogits is not None:
        a.dlogits = _matrix(dlogits, "dlogits")
    return a, m.rows


def token_logprob(logits, targets=None, top_k: int = 0, g_logp=None, g_entropy=None, g_lse=None, dlogits=None,
                  stream=None) -> TokenLogprob:
    """Log probabilities of ``targets`` (int64, negative: none) under ``logits``
    (rows x vocabulary), with entropy, lse and the ``top_k`` best alternatives.
    With any of the weights ``g_*`` (float32, one a row) the gradient of
    sum(g_logp logp + g_entropy entropy + g_lse lse) comes from the same call,
    in ``dlogits`` (a new tensor if None; ``logits`` itself is allowed)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return token_logprob(logits, targets, top_k, g_logp, g_entropy, g_lse, dlogits)
    lib = _L.load_library()
    if dlogits is None and (g_logp is not None or g_entropy is not None or g_lse is not None):
        dlogits = logits.new_empty(logits.shape)
    a, n = _logprob_args(logits, targets, g_logp, g_entropy, g_lse, dlogits)
    lead, device = logits.shape[:-1], logits.device
    entropy, lse = torch.empty(lead, dtype=torch.float32, device=device), torch.empty(lead, dtype=torch.float32, device=device)
    a.entropy, a.lse = entropy.data_ptr(), lse.data_ptr()
    logp = top_logp = top_index = None
    if targets is not None:
        logp = torch.empty(lead, dtype=torch.float32, device=device)
        a.logp = logp.data_ptr()
    a.top_k = top_k
    if top_k > 0:
        top_logp = torch.empty((*lead, top_k), dtype=torch.float32, device=device)
        top_index = torch.empty((*lead, top_k), dtype=torch.int64, device=device)
        a.top_logp, a.top_index = top_logp.data_ptr(), top_index.data_ptr()
    st = lib.lm_token_logprob(a, _stream_of(logits))
    if st:
        _L._check(lib, st, "lm_token_logprob")
    return TokenLogprob(logp, entropy, lse, top_logp, top_index, dlogits)


def token_logprob_grad(logits, targets, lse, entropy, g_logp, g_entropy=None, g_lse=None, dlogits=None, stream=None):
    """The gradient of ``token_logprob`` for weights known after the forward
    call, from its ``lse`` and (with ``g_entropy``) ``entropy``."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return token_logprob_grad(logits, targets, lse, entropy, g_logp, g_entropy, g_lse, dlogits)
    lib = _L.load_library()
    if dlogits is None:
        dlogits = logits.new_empty(logits.shape)
    a, n = _logprob_args(logits, targets, g_logp, g_entropy, g_lse, dlogits)
    a.lse = _array(lse, n, torch.float32, "lse")
    a.entropy = _array(entropy, n, torch.float32, "entropy")
    st = lib.lm_token_logprob_grad(a, _stream_of(logits))
    if st:
        _L._check(lib, st, "lm_token_logprob_grad")
    return dlogits


class LinearLogprob(NamedTuple):
    """``logp``, ``entropy`` and ``lse``, one entry a row (``logp`` None without
    targets); the gradients ``dh`` and ``dweight`` None without weights."""
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    lse: torch.Tensor
    dh: Optional[torch.Tensor]
    dweight: Optional[torch.Tensor]


def _linear_logprob(fn, lib, h, weight, targets, logp, entropy, lse, g_logp, g_entropy, g_lse, dh, dweight, accumulate):
    mh = _matrix_fields(h, "h")
    n = mh[1]
    floats = [_array(t, n, torch.float32, what) or 0 if t is not None else 0
              for t, what in ((logp, "logp"), (entropy, "entropy"), (lse, "lse"), (g_logp, "g_logp"), (g_entropy, "g_entropy"), (g_lse, "g_lse"))]
    a = _pack_linear_logprob(*mh, *_matrix_fields(weight, "weight"), _array(targets, n, torch.int64, "targets") or 0, *floats,
                             *(_matrix_fields(dh, "dh") if dh is not None else _NO_MATRIX),
                             *(_matrix_fields(dweight, "dweight") if dweight is not None else _NO_MATRIX), 1 if accumulate else 0)
    need = lib.lm_linear_logprob_workspace(a)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    st = getattr(lib, fn)(a, ws.data_ptr() if need else None, need, _stream_of(h))
    if st:
        _L._check(lib, st, fn)


def _gradients(h, weight, dh, dweight, accumulate, none):
    """What receives the gradients: new tensors for None (None with ``none``), None for False."""
    if accumulate and (dweight is None or dweight is False):
        raise ValueError("accumulate adds to dweight: give it")
    made = lambda t, like: None if t is False or (none and t is None) else torch.empty(like.shape, dtype=like.dtype, device=like.device) if t is None else t  # noqa: E731
    return made(dh, h), made(dweight, weight)


def linear_logprob(h, weight, targets=None, g_logp=None, g_entropy=None, g_lse=None, dh=None, dweight=None,
                   accumulate: bool = False, stream=None) -> LinearLogprob:
    """``token_logprob`` of the logits h weight^T (bf16, rows x width and
    vocabulary x width), which are never formed.  With any of the weights
    ``g_*`` the gradients of sum(g_logp logp + g_entropy entropy + g_lse lse) by
    h and weight come from the same call, in ``dh`` and ``dweight`` (new tensors
    if None, not computed if False; ``dweight``, bf16 or fp32, has its gradient
    added with ``accumulate``)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return linear_logprob(h, weight, targets, g_logp, g_entropy, g_lse, dh, dweight, accumulate)
    lib = _L.load_library()
    dh, dweight = _gradients(h, weight, dh, dweight, accumulate, g_logp is None and g_entropy is None and g_lse is None)
    lead, device = h.shape[:-1], h.device
    entropy, lse = torch.empty(lead, dtype=torch.float32, device=device), torch.empty(lead, dtype=torch.float32, device=device)
    logp = torch.empty(lead, dtype=torch.float32, device=device) if targets is not None else None
    _linear_logprob("lm_linear_logprob", lib, h, weight, targets, logp, entropy, lse, g_logp, g_entropy, g_lse, dh, dweight, accumulate)
    return LinearLogprob(logp, entropy, lse, dh, dweight)


def linear_logprob_grad(h, weight, targets, lse, entropy, g_logp, g_entropy=None, g_lse=None, dh=None, dweight=None,
                        accumulate: bool = False, stream=None):
    """(dh, dweight) of ``linear_logprob`` for weights known after the forward
    call, from its ``lse`` and (with ``g_entropy``) ``entropy``; None for what
    is False."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return linear_logprob_grad(h, weight, targets, lse, entropy, g_logp, g_entropy, g_lse, dh, dweight, accumulate)
    lib = _L.load_library()
    dh, dweight = _gradients(h, weight, dh, dweight, accumulate, False)
    _linear_logprob("lm_linear_logprob_grad", lib, h, weight, targets, None, entropy, lse, g_logp, g_entropy, g_lse, dh, dweight, accumulate)
    return dh, dweight


def rotary_frequencies(dims: int, base: float = 10000.0, factor: float = 1.0, original: int = 0, low: float = 1.0,
                       high: float = 4.0):
    """Angles a position, one for each of dims / 2 pairs (float64, CPU):
    base^(-2 j / dims), for contexts ``factor`` times as long divided by it.
    With ``original`` (positions the model was trained on) only the slow ones
    are: those that turn at least ``high`` times within them stay, those that
    turn at most ``low`` times are divided, the others lie between, by their
    number of turns."""
    if dims < 0 or dims % 2:
        raise ValueError(f"dims {dims} is not even")
    if not base > 0 or not factor > 0 or (original and not high > low):
        raise ValueError("base and factor are positive, and high is above low")
    f = base ** (-torch.arange(0, dims, 2, dtype=torch.float64) / max(dims, 1))
    if not original:
        return f / factor
    keep = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
    return f * keep + f / factor * (1 - keep)


def rotary_table(positions: int, frequencies, amplitude: float = 1.0, device="cuda"):
    """The table that ``qk_rotary`` reads: amplitude times cosine and sine of
    position times frequency, positions x dims / 2 x 2, float32 (angles in 64
    bits, rounded once)."""
    f = torch.as_tensor(frequencies, dtype=torch.float64, device=device)
    a = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * f
    return torch.stack((a.cos(), a.sin()), dim=-1).mul_(amplitude).float()


class QkRotary(NamedTuple):
    q: torch.Tensor
    k: Optional[torch.Tensor]


class QkRotaryGrad(NamedTuple):
    """Gradients of the queries, of the keys (None without them) and of their
    gains (None where there is no norm or none was wanted)."""
    dq: torch.Tensor
    dk: Optional[torch.Tensor]
    dq_weight: Optional[torch.Tensor]
    dk_weight: Optional[torch.Tensor]


def _heads(t, what: str):
    """lm_heads' fields of a tensor (.., heads, dim): the leading dimensions fold
    into tokens of one pitch."""
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what}: unsupported dtype {t.dtype}")
    shape = t.shape
    if len(shape) != 3:
        if len(shape) < 2:
            raise ValueError(f"{what}: expected (.., heads, dim)")
        try:
            t = t.view(math.prod(shape[:-2]), *shape[-2:])
        except RuntimeError:
            raise ValueError(f"{what}: the leading dimensions do not fold into tokens of one pitch") from None
        shape = t.shape
    tokens, heads, dim = shape
    by_token, by_head, one = t.stride()
    if one != 1 and dim > 1 and tokens > 0 and heads > 0:
        raise ValueError(f"{what}: the last dimension must have stride 1")
    return t.data_ptr(), tokens, heads, dim, by_token, by_head, code


def _rotary_tail(tokens: int, positions, table, norm, eps, interleaved):
    """The fields of lm_qk_rotary_args after its parts."""
    at = rows = turned = where = 0
    if table is not None:
        if table.dtype != torch.float32:
            raise TypeError(f"table: expected float32, got {table.dtype}")
        if table.dim() != 3 or table.shape[2] != 2 or not table.is_contiguous():
            raise ValueError("table: expected positions x dims / 2 x 2, contiguous")
        if positions is None:
            raise ValueError("a table goes with positions")
        at = _array(positions, tokens, torch.int64, "positions")
        rows, pairs, _ = table.shape
        where, turned = table.data_ptr(), 2 * pairs
    return at, where, rows, turned, 1 if norm else 0, 1 if interleaved else 0, eps


def qk_rotary(q, k, positions, table, q_weight=None, k_weight=None, norm: bool = True, eps: float = 1e-6,
              interleaved: bool = False, q_out=None, k_out=None, stream=None) -> QkRotary:
    """Queries and keys (.., heads, dim; k may be None) with each head's RMS norm
    and gain (``norm``) and the rotation by position: ``positions`` (int64, one a
    token) into ``table`` (``rotary_table``; its width says how many channels
    turn; None for none).  ``q_out`` and ``k_out`` receive the results (new
    tensors if None; q and k themselves are allowed)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return qk_rotary(q, k, positions, table, q_weight, k_weight, norm, eps, interleaved, q_out, k_out)
    lib = _L.load_library()
    hq = _heads(q, "q")
    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else q_out
    fields = [*hq, *_heads(q_out, "q_out"), *_NO_HEADS, *(_vector_fields(q_weight, "q_weight") if q_weight is not None else _NO_TENSOR), *_NO_TENSOR]
    if k is not None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None else k_out
        fields += [*_heads(k, "k"), *_heads(k_out, "k_out"), *_NO_HEADS, *(_vector_fields(k_weight, "k_weight") if k_weight is not None else _NO_TENSOR),
                   *_NO_TENSOR]
    elif k_weight is not None or k_out is not None:
        raise ValueError("k_weight or k_out without k")
    else:
        fields += _NO_PART
    st = lib.lm_qk_rotary(_pack_qk_rotary(*fields, *_rotary_tail(hq[1], positions, table, norm, eps, interleaved)), _stream_of(q))
    if st:
        _L._check(lib, st, "lm_qk_rotary")
    return QkRotary(q_out, k_out)


def qk_rotary_grad(dq, dk, positions, table, q=None, k=None, q_weight=None, k_weight=None, norm: bool = True,
                   eps: float = 1e-6, interleaved: bool = False, dq_out=None, dk_out=None, dweight: bool = True,
                   stream=None) -> QkRotaryGrad:
    """The gradient of ``qk_rotary``.  q and k, the forward call's inputs, are
    read with the norm only.  ``dq_out`` and ``dk_out`` receive the gradients
    (new tensors if None; dq and dk themselves are allowed).  The gains'
    gradients have the dtype of the gains, float32 where there are none."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return qk_rotary_grad(dq, dk, positions, table, q, k, q_weight, k_weight, norm, eps, interleaved, dq_out,
                                  dk_out, dweight)
    lib = _L.load_library()
    tokens = _heads(dq, "dq")[1]
    gains = [None, None]
    outs = [dq_out, dk_out]
    fields = []
    for i, (d, x, w) in enumerate(((dq, q, q_weight), (dk, k, k_weight))):
        if d is None:
            if w is not None or outs[i] is not None or x is not None:
                raise ValueError("keys, their gain or gradient without dk")
            fields += _NO_PART
            continue
        if outs[i] is None:
            outs[i] = torch.empty(d.shape, dtype=d.dtype, device=d.device)
        if norm:
            if x is None:
                raise ValueError("the gradient of the norm reads q and k")
            if dweight:
                gains[i] = torch.empty(d.shape[-1], dtype=w.dtype if w is not None else torch.float32, device=d.device)
        fields += [*(_heads(x, "q" if i == 0 else "k") if norm else _NO_HEADS), *_heads(d, "dq" if i == 0 else "dk"),
                   *_heads(outs[i], "dq_out" if i == 0 else "dk_out"),
                   *(_vector_fields(w, "q_weight" if i == 0 else "k_weight") if w is not None else _NO_TENSOR),
                   *(_vector_fields(gains[i], "dweight") if gains[i] is not None else _NO_TENSOR)]
    a = _pack_qk_rotary(*fields, *_rotary_tail(tokens, positions, table, norm, eps, interleaved))
    need = lib.lm_qk_rotary_grad_workspace(a) if norm and dweight else 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    st = lib.lm_qk_rotary_grad(a, ws.data_ptr() if need else None, need, _stream_of(dq))
    if st:
        _L._check(lib, st, "lm_qk_rotary_grad")
    return QkRotaryGrad(outs[0], outs[1], gains[0], gains[1])
