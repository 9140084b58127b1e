"""Operators on a caller's own matrices: products with 8-bit weights, and rules on logits.

As in translator.py, every call only checks and allocates torch tensors, passes raw pointers and the current HIP stream of the
tensors' GPU to the matching ``onmt_*`` function and returns tensors. Matrices are fp32, bf16 or fp16 with contiguous
columns and any row stride.
"""

import ctypes
import functools

import torch

from . import _lib
from ._lib import OnmtLogitRules, check

_TYPES = {torch.float32: _lib.ONMT_F32, torch.bfloat16: _lib.ONMT_BF16, torch.float16: _lib.ONMT_F16}


def _on_gpu(name, t, device=None):
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise ValueError(f"{name} must be a tensor on the GPU")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the other tensors on {device}")


def _matrix(name, t, device=None, rows=None, cols=None, dtypes=None):
    """The row stride of a matrix the library can take."""
    _on_gpu(name, t, device)
    if t.dim() != 2 or t.shape[0] < 1 or t.shape[1] < 1:
        raise ValueError(f"{name} must be a matrix with at least one row and column, got {tuple(t.shape)}")
    if t.dtype not in (dtypes or _TYPES):
        raise ValueError(f"{name} has type {t.dtype}")
    if (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected ({rows or 'any'}, {cols or 'any'})")
    ld = t.stride(0) if t.shape[0] > 1 else t.shape[1]
    if (t.shape[1] > 1 and t.stride(1) != 1) or ld < t.shape[1]:
        raise ValueError(f"{name} needs contiguous columns and rows that do not overlap, got strides {t.stride()}")
    return ld


def _vector(name, t, n, dtype, device):
    _on_gpu(name, t, device)
    if t.dtype != dtype or t.dim() != 1 or (n is not None and t.shape[0] != n) or (t.shape[0] > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous {dtype} vector" + (f" of {n}" if n is not None else ""))


# A decoding program makes these calls every step: sizes that depend on nothing else are asked once, and the stream's handle is
# read without making a torch.cuda.Stream (9 of the 17 us that a small call took on the host).
@functools.lru_cache(maxsize=4096)
def _bytes_of(query, *sizes):
    return getattr(_lib.load(), query)(*sizes)


def _call(device, function, *args):
    """The library call with the tensors' GPU as the current one, on that GPU's current stream."""
    if device.index == torch.cuda.current_device():
        check(function(*args, torch._C._cuda_getCurrentRawStream(device.index)))
    else:
        with torch.cuda.device(device):
            check(function(*args, torch._C._cuda_getCurrentRawStream(device.index)))


class F8Weights:
    """A weight matrix [rows, cols] held as e4m3 values with a power of two per row and block of 128 columns."""

    def __init__(self, w):
        ld = _matrix("w", w)
        self.rows, self.cols = w.shape
        self.device = w.device
        n = _bytes_of("onmt_f8_bytes", self.rows, self.cols)
        self.buf = torch.empty(n, dtype=torch.uint8, device=w.device)
        _call(w.device, _lib.load().onmt_f8_pack, w.data_ptr(), _TYPES[w.dtype], ld, self.rows, self.cols, self.buf.data_ptr(), n)

    def values(self):
        """The fp32 values [rows, cols] that the weights stand for."""
        out = torch.empty(self.rows, self.cols, dtype=torch.float32, device=self.device)
        _call(self.device, _lib.load().onmt_f8_unpack, self.buf.data_ptr(), self.buf.numel(), self.rows, self.cols,
              out.data_ptr(), self.cols)
        return out

    def linear(self, x, bias=None, out_dtype=torch.float32, out=None):
        """x [M, cols], rounded to 8 bits like the weights, times the weights' transpose, plus bias [rows] (fp32): [M, rows] of
        out_dtype, or written to out."""
        device = self.device
        ldx = _matrix("x", x, device, cols=self.cols)
        M = x.shape[0]
        if bias is not None:
            _vector("bias", bias, self.rows, torch.float32, device)
        if out is None:
            if out_dtype not in _TYPES:
                raise ValueError(f"out_dtype is {out_dtype}")
            out = torch.empty(M, self.rows, dtype=out_dtype, device=device)
            ld = self.rows
        else:
            ld = _matrix("out", out, device, M, self.rows)
        kind = _TYPES[out.dtype]
        n = _bytes_of("onmt_f8_linear_ws_bytes", M, self.cols)
        ws = torch.empty(n, dtype=torch.uint8, device=device) if n else None
        _call(device, _lib.load().onmt_f8_linear, x.data_ptr(), _TYPES[x.dtype], ldx, M, self.buf.data_ptr(), self.buf.numel(),
              self.rows, self.cols, bias.data_ptr() if bias is not None else None, out.data_ptr(), kind, ld,
              ws.data_ptr() if n else None, n)
        return out


class LogitRules:
    """The rules of onmt_logit_rules. The tensors are kept and read by every call, so a step loop appends to `history` and
    `history_len` in place.

    history [N, T] int32 with history_len [N] int32; repetition, presence, frequency [N] fp32; no_repeat_ngram; bias_ids and
    bias [N, n] (int32, fp32; ids outside the vocabulary are ignored, the last entry of an id counts); mask [tables, words] int32
    (bit v & 31 of word v >> 5: token v is allowed) with mask_row [N] int32 (negative: no mask), or a table per row without it.
    """

    def __init__(self, history=None, history_len=None, repetition=None, presence=None, frequency=None, no_repeat_ngram=0,
                 bias_ids=None, bias=None, mask=None, mask_row=None):
        given = [t for t in (history, history_len, repetition, presence, frequency, bias_ids, bias, mask, mask_row)
                 if t is not None]
        for t in given:
            _on_gpu("a tensor of the rules", t, given[0].device)
        self.device = given[0].device if given else None
        self.tensors = given
        self.rows = None
        c = self.c = OnmtLogitRules()

        def rows(name, t, n):
            if self.rows not in (None, n):
                raise ValueError(f"{name} is for {n} rows, the tensors before it for {self.rows}")
            self.rows = n

        if (history is None) != (history_len is None):
            raise ValueError("history and history_len come together")
        if (bias_ids is None) != (bias is None):
            raise ValueError("bias_ids and bias come together")
        if mask_row is not None and mask is None:
            raise ValueError("mask_row without mask")
        if history is not None and history.shape[-1] > 0:
            c.history_stride = _matrix("history", history, dtypes=(torch.int32,))
            c.history, c.max_history = history.data_ptr(), history.shape[1]
            rows("history", history, history.shape[0])
            _vector("history_len", history_len, self.rows, torch.int32, self.device)
            c.history_len = history_len.data_ptr()
        for name, t in (("repetition", repetition), ("presence", presence), ("frequency", frequency)):
            if t is not None:
                _vector(name, t, self.rows, torch.float32, self.device)
                rows(name, t, t.shape[0])
                setattr(c, name, t.data_ptr())
        c.no_repeat_ngram = no_repeat_ngram
        if bias is not None and bias.shape[-1] > 0:
            c.bias_stride = _matrix("bias_ids", bias_ids, dtypes=(torch.int32,))
            rows("bias_ids", bias_ids, bias_ids.shape[0])
            if _matrix("bias", bias, rows=self.rows, cols=bias_ids.shape[1], dtypes=(torch.float32,)) != c.bias_stride:
                raise ValueError("bias_ids and bias have different row strides")
            c.bias_ids, c.bias, c.n_bias = bias_ids.data_ptr(), bias.data_ptr(), bias.shape[1]
        if mask is not None:
            c.mask_stride = _matrix("mask", mask, dtypes=(torch.int32,))
            c.mask, c.n_masks = mask.data_ptr(), mask.shape[0]
            if mask_row is not None:
                _vector("mask_row", mask_row, self.rows, torch.int32, self.device)
                rows("mask_row", mask_row, mask_row.shape[0])
                c.mask_row = mask_row.data_ptr()
            else:
                rows("mask", mask, mask.shape[0])
        self.words = mask.shape[1] if mask is not None else None


def constrain(logits, rules=None, mode=0, K=1, out=None):
    """(out, ids, lse) of logits [N, V] under the rules (onmt_constrain). mode 0: out [N, V] fp32 log-probabilities; 1: out and
    ids [N, K] of the K largest; 2: out [N, V] = the logits under the rules, in their own type. What a mode does not give is None.
    out: where to write modes 0 and 2, the logits themselves for example."""
    ld = _matrix("logits", logits)
    N, V = logits.shape
    device = logits.device
    if mode not in (0, 1, 2):
        raise ValueError("mode must be 0 (log-probs), 1 (top-K) or 2 (logits)")
    ref = None
    if rules is not None:
        if rules.device is not None and rules.device != device:
            raise ValueError(f"the rules are on {rules.device}, the logits on {device}")
        if rules.rows not in (None, N):
            raise ValueError(f"the rules are for {rules.rows} rows, the logits have {N}")
        if rules.words is not None and rules.words < (V + 31) // 32:
            raise ValueError(f"a mask of {rules.words} words does not cover {V} tokens")
        ref = ctypes.byref(rules.c)
    out_dtype = logits.dtype if mode == 2 else torch.float32
    ids = lse = ws = None
    n = 0
    if out is not None:
        if mode == 1:
            raise ValueError("out is for modes 0 and 2")
        ld_out = _matrix("out", out, device, N, V, (out_dtype,))
    else:
        ld_out = K if mode == 1 else V
        out = torch.empty(N, max(ld_out, 0), dtype=out_dtype, device=device)
    if mode != 2:
        n = _bytes_of("onmt_constrain_ws_bytes", N, V, mode, K)
        ws = torch.empty(n, dtype=torch.uint8, device=device)
        lse = torch.empty(N, dtype=torch.float32, device=device)
        if mode == 1:
            ids = torch.empty(N, max(K, 0), dtype=torch.int32, device=device)
    _call(device, _lib.load().onmt_constrain, ref, logits.data_ptr(), _TYPES[logits.dtype], ld, N, V, mode, K, out.data_ptr(),
          ld_out, ids.data_ptr() if ids is not None else None, lse.data_ptr() if lse is not None else None,
          ws.data_ptr() if n else None, n)
    return out, ids, lse
