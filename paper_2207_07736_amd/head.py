"""Thin Python binding of the output head's operators (rlsim_head_* of
include/rlsim.h): argument marshalling only.

``Head`` draws actions or tokens from rows of logits and distils a student's rows
from a teacher's top logits.  torch is used for device memory, and so that
``Head.distill_loss`` can take part in its backward pass.
"""
from __future__ import annotations

import ctypes

from .rlsim import RLSIM_BF16, RLSIM_F16, RLSIM_F32, RLSIM_OK, RlsimError, lib


class rlsim_sample(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("logits", ctypes.c_void_p), ("rows", ctypes.c_uint32),
                ("vocab", ctypes.c_uint32), ("row_stride", ctypes.c_uint64), ("u", ctypes.c_void_p),
                ("temperature", ctypes.c_float), ("top_k", ctypes.c_uint32), ("top_p", ctypes.c_float),
                ("min_p", ctypes.c_float), ("temperature_rows", ctypes.c_void_p), ("top_k_rows", ctypes.c_void_p),
                ("top_p_rows", ctypes.c_void_p), ("min_p_rows", ctypes.c_void_p), ("token", ctypes.c_void_p),
                ("logp", ctypes.c_void_p)]


class rlsim_distill(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("logits", ctypes.c_void_p), ("rows", ctypes.c_uint32),
                ("vocab", ctypes.c_uint32), ("row_stride", ctypes.c_uint64), ("teacher_dtype", ctypes.c_int),
                ("teacher", ctypes.c_void_p), ("teacher_stride", ctypes.c_uint64), ("index_bytes", ctypes.c_int),
                ("index", ctypes.c_void_p), ("index_stride", ctypes.c_uint64), ("k", ctypes.c_uint32),
                ("temperature", ctypes.c_float), ("rest", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("loss", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("grad_stride", ctypes.c_uint64)]


lib.rlsim_head_create.argtypes = [ctypes.c_uint32, ctypes.c_uint32, ctypes.c_void_p, ctypes.POINTER(ctypes.c_void_p)]
lib.rlsim_head_create.restype = ctypes.c_int
lib.rlsim_head_sample.argtypes = [ctypes.c_void_p, ctypes.POINTER(rlsim_sample)]
lib.rlsim_head_sample.restype = ctypes.c_int
lib.rlsim_head_distill.argtypes = [ctypes.c_void_p, ctypes.POINTER(rlsim_distill)]
lib.rlsim_head_distill.restype = ctypes.c_int
lib.rlsim_head_destroy.argtypes = [ctypes.c_void_p]
lib.rlsim_head_destroy.restype = ctypes.c_int
lib.rlsim_head_last_error.argtypes = [ctypes.c_void_p]
lib.rlsim_head_last_error.restype = ctypes.c_char_p


def _check_head(rc: int, h) -> None:
    if rc != RLSIM_OK:
        msg = lib.rlsim_head_last_error(h)
        raise RlsimError(rc, msg.decode() if msg else "rlsim error")


def rlsim_head_last_error(h=None) -> str:
    return lib.rlsim_head_last_error(h).decode()


def rlsim_head_create(max_rows: int, max_vocab: int, stream=None) -> ctypes.c_void_p:
    """A head's handle; ``stream`` is a torch.cuda.Stream, a raw hipStream_t int, or
    None for the default stream."""
    if stream is not None:
        stream = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    h = ctypes.c_void_p()
    _check_head(lib.rlsim_head_create(int(max_rows), int(max_vocab), stream, ctypes.byref(h)), None)
    return h


def rlsim_head_sample(h, args: rlsim_sample) -> None:
    _check_head(lib.rlsim_head_sample(h, ctypes.byref(args)), h)


def rlsim_head_distill(h, args: rlsim_distill) -> None:
    _check_head(lib.rlsim_head_distill(h, ctypes.byref(args)), h)


def rlsim_head_destroy(h) -> None:
    if h:
        _check_head(lib.rlsim_head_destroy(h), None)


class Head:
    """Owning wrapper of one head handle: operators on rows of logits for up to
    ``max_rows`` rows of up to ``max_vocab`` entries.  Tensors are on the device the
    handle was created on, and are used on the handle's stream: work that makes or
    frees them elsewhere has to be ordered with it."""

    def __init__(self, max_rows: int, max_vocab: int, stream=None):
        import torch
        self.h = None
        self._dtypes = {torch.float32: RLSIM_F32, torch.bfloat16: RLSIM_BF16, torch.float16: RLSIM_F16}
        self._index = {torch.int32: 4, torch.int64: 8}
        self._torch = torch
        self.device = torch.device("cuda", torch.cuda.current_device())
        self.max_rows, self.max_vocab = int(max_rows), int(max_vocab)
        self.h = rlsim_head_create(max_rows, max_vocab, stream)

    def close(self):
        if self.h:
            h, self.h = self.h, None
            rlsim_head_destroy(h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, name, t, rows=None, columns=None):
        """A 2-d tensor whose rows are consecutive elements, and its row stride."""
        if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (columns is not None and t.shape[1] != columns):
            raise ValueError(f"{name} must be 2-d" + ("" if rows is None else f", [{rows}, {columns or 'k'}]"))
        if t.device != self.device:
            raise ValueError(f"{name} must be on {self.device}")
        stride = t.stride(0) if t.shape[0] > 1 else t.shape[1]
        if t.shape[1] > 1 and t.stride(1) != 1 or stride < t.shape[1]:
            raise ValueError(f"{name} must hold each row in consecutive elements, rows apart")
        return t.data_ptr(), stride

    def _vector(self, name, t, rows, dtype):
        """The address of a [rows] tensor, None for None."""
        if t is None:
            return None
        if t.dtype != dtype or t.dim() != 1 or t.shape[0] != rows or (rows > 1 and t.stride(0) != 1) or t.device != self.device:
            raise ValueError(f"{name} must be {dtype}, [{rows}], contiguous, on {self.device}")
        return t.data_ptr()

    def _dtype(self, name, t):
        try:
            return self._dtypes[t.dtype]
        except KeyError:
            raise ValueError(f"{name} must be float32, bfloat16 or float16") from None

    def sample(self, logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, logp: bool = False):
        """Draw one entry of each row of ``logits`` [rows, vocab] from the uniform
        numbers ``u`` [rows] (float32).  Each setting is a number, or a [rows] tensor
        (float32; top_k: int32).  Returns the int32 tokens, or with ``logp`` also
        their float32 log-probabilities among the entries that the filters keep."""
        torch = self._torch
        a = rlsim_sample()
        a.dtype = self._dtype("logits", logits)
        a.logits, a.row_stride = self._rows("logits", logits)
        rows, a.vocab = logits.shape
        a.rows = rows
        if u is None:
            raise ValueError("u is needed")
        a.u = self._vector("u", u, rows, torch.float32)
        if torch.is_tensor(temperature):
            a.temperature_rows = self._vector("temperature", temperature, rows, torch.float32)
        else:
            a.temperature = temperature
        if torch.is_tensor(top_k):
            a.top_k_rows = self._vector("top_k", top_k, rows, torch.int32)
        else:
            if top_k < 0 or top_k > 0xFFFFFFFF:
                raise ValueError("top_k must be >= 0")
            a.top_k = top_k
        if torch.is_tensor(top_p):
            a.top_p_rows = self._vector("top_p", top_p, rows, torch.float32)
        else:
            a.top_p = top_p
        if torch.is_tensor(min_p):
            a.min_p_rows = self._vector("min_p", min_p, rows, torch.float32)
        else:
            a.min_p = min_p
        token = torch.empty(rows, dtype=torch.int32, device=self.device)
        a.token = token.data_ptr()
        p = None
        if logp:
            p = torch.empty(rows, dtype=torch.float32, device=self.device)
            a.logp = p.data_ptr()
        rlsim_head_sample(self.h, a)
        return (token, p) if logp else token

    def distill(self, logits, teacher, index, temperature: float = 1.0, rest=None, weight=None, loss: bool = True, grad=True):
        """Distil rows of student ``logits`` [rows, vocab] from a teacher's top logits
        ``teacher`` [rows, k] at the entries ``index`` [rows, k] (int32 or int64; outside
        the row: an empty slot), optionally with ``rest`` [rows], the log of the sum of
        exp(t / temperature) over what it does not list.  Returns the float32 losses
        [rows] and the gradient of sum(weight * loss) in the logits' type; ``loss``
        or ``grad`` False leaves that one out.  ``grad`` may be a tensor to write to,
        the logits themselves among them."""
        torch = self._torch
        a = rlsim_distill()
        a.dtype = self._dtype("logits", logits)
        a.logits, a.row_stride = self._rows("logits", logits)
        rows, a.vocab = logits.shape
        a.rows = rows
        a.teacher_dtype = self._dtype("teacher", teacher)
        a.teacher, a.teacher_stride = self._rows("teacher", teacher, rows)
        if index.dtype not in self._index:
            raise ValueError("index must be int32 or int64")
        a.k = teacher.shape[1]
        a.index_bytes = self._index[index.dtype]
        a.index, a.index_stride = self._rows("index", index, rows, a.k)
        a.temperature = temperature
        a.rest = self._vector("rest", rest, rows, torch.float32)
        a.weight = self._vector("weight", weight, rows, torch.float32)
        losses = None
        if loss:
            losses = torch.empty(rows, dtype=torch.float32, device=self.device)
            a.loss = losses.data_ptr()
        out = None
        if grad is not False:
            if grad is True:
                out = torch.empty(logits.shape, dtype=logits.dtype, device=self.device)
            else:
                out = grad
                if out.dtype != logits.dtype:
                    raise ValueError("grad must have the logits' type")
            a.grad, a.grad_stride = self._rows("grad", out, rows, logits.shape[1])
        rlsim_head_distill(self.h, a)
        if loss and out is not None:
            return losses, out
        return losses if loss else out

    def distill_loss(self, logits, teacher, index, temperature: float = 1.0, rest=None):
        """The losses of ``distill`` [rows], differentiable with respect to ``logits``
        (the teacher is a constant)."""
        return _distill_function(self._torch).apply(self, logits, teacher, index, temperature, rest)


_function = None


def _distill_function(torch):
    """The autograd function behind Head.distill_loss, made on first use: forward
    computes the losses, backward the gradient from the losses' own."""
    global _function
    if _function is None:
        class DistillLoss(torch.autograd.Function):
            @staticmethod
            def forward(ctx, head, logits, teacher, index, temperature, rest):
                ctx.head, ctx.temperature = head, temperature
                ctx.save_for_backward(logits, teacher, index, *(() if rest is None else (rest,)))
                return head.distill(logits, teacher, index, temperature, rest, grad=False)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, g):
                logits, teacher, index, *rest = ctx.saved_tensors
                out = ctx.head.distill(logits, teacher, index, ctx.temperature, rest[0] if rest else None,
                                       weight=g.contiguous(), loss=False)
                return None, out, None, None, None, None

        _function = DistillLoss
    return _function
