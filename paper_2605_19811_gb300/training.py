"""Training-step operators next to the optimizer (the second half of
``include/lionmuon.h``): token log probabilities with entropy, top alternatives
and gradient; RMS norm with the residual's addition, an 8-bit output and
gradient; 8-bit activation checkpoints and the weight gradient of a linear
layer taken from them.

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


def _matrix(t, what: str) -> LmMatrix:
    """lm_matrix of a tensor (a vector is one row)."""
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
    return LmMatrix(t.data_ptr(), rows, cols, ld if rows > 1 else cols, code)


def _vector(t, what: str) -> LmTensor:
    if t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous vector")
    return LmTensor(t.data_ptr(), 1, t.shape[0], _dtype(t))


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
    x (at least) rows; ``cols`` channels; ``format`` "i8" or "e4m3"."""

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

    def desc(self) -> LmCheckpoint8:
        codes, scales = self.codes, self.scales
        rows, pitch = codes.shape
        groups, lds = scales.shape
        # (one row of a wider buffer keeps its buffer's pitch, as several do)
        return LmCheckpoint8(codes.data_ptr(), scales.data_ptr(), rows, self.cols, codes.stride(0) if rows > 1 else max(codes.stride(0), pitch),
                             scales.stride(0) if groups > 1 else lds, FORMATS[self.format])

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
