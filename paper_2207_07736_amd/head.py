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
    rc = lib.rlsim_head_sample(h, ctypes.byref(args))
    if rc:
        _check_head(rc, h)


def rlsim_head_distill(h, args: rlsim_distill) -> None:
    rc = lib.rlsim_head_distill(h, ctypes.byref(args))
    if rc:
        _check_head(rc, h)


def rlsim_head_destroy(h) -> None:
    if h:
        _check_head(lib.rlsim_head_destroy(h), None)


class Head:
    """Owning wrapper of one head handle: operators on rows of logits for up to
    ``max_rows`` rows (none among them) of up to ``max_vocab`` entries.  Tensors are on the device the
    handle was created on, and are used on the handle's stream: work that makes or
    frees them elsewhere has to be ordered with it (``distill_loss`` orders itself).  That
    holds for the returned tensors too, which torch allocates for its current stream.
    All calls of a handle, and all replays of graphs that captured some, have to be
    ordered with one another: graphs that may run at the same time need a Head each, and
    none is replayed once its Head is closed."""

    def __init__(self, max_rows: int, max_vocab: int, stream=None):
        import torch
        self.h = None
        self._dtypes = {torch.float32: RLSIM_F32, torch.bfloat16: RLSIM_BF16, torch.float16: RLSIM_F16}
        self._index = {torch.int32: 4, torch.int64: 8}
        self._torch, self._tensor, self._empty = torch, torch.Tensor, torch.empty
        self._written = torch.autograd.graph.increment_version
        self._f32, self._i32 = torch.float32, torch.int32
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._ordinal = self.device.index
        self.max_rows, self.max_vocab = int(max_rows), int(max_vocab)
        if stream is None or not hasattr(stream, "cuda_stream"):
            stream = (torch.cuda.ExternalStream(int(stream), device=self.device) if stream
                      else torch.cuda.default_stream(self.device))
        self._stream = stream
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
        """The address of a 2-d tensor whose rows are consecutive elements, its shape and
        its row stride."""
        shape = t.shape
        if len(shape) != 2 or (rows is not None and shape[0] != rows) or (columns is not None and shape[1] != columns):
            raise ValueError(f"{name} must be 2-d" + ("" if rows is None else f", [{rows}, {columns or 'k'}]"))
        if t.get_device() != self._ordinal:
            raise ValueError(f"{name} must be on {self.device}")
        n, width = shape
        if t.is_contiguous():
            return t.data_ptr(), n, width, width
        stride, step = t.stride()
        stride = stride if n > 1 else width
        if (width > 1 and step != 1) or stride < width:
            raise ValueError(f"{name} must hold each row in consecutive elements, rows apart")
        return t.data_ptr(), n, width, stride

    def _vector(self, name, t, rows, dtype):
        """The address of a [rows] tensor, None for None."""
        if t is None:
            return None
        if t.dtype != dtype or t.shape != (rows,) or not t.is_contiguous() or t.get_device() != self._ordinal:
            raise ValueError(f"{name} must be {dtype}, [{rows}], contiguous, on {self.device}")
        return t.data_ptr()

    def _setting(self, name, value, rows, dtype):
        """A setting as a number for the call and an address of [rows] numbers, one of them."""
        if isinstance(value, self._tensor):
            return 0, self._vector(name, value, rows, dtype)
        return value, None

    def _dtype(self, name, t):
        try:
            return self._dtypes[t.dtype]
        except KeyError:
            raise ValueError(f"{name} must be float32, bfloat16 or float16") from None

    def sample(self, logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, logp: bool = False):
        """Draw one entry of each row of ``logits`` [rows, vocab] from the uniform
        numbers ``u`` [rows] (float32).  Each setting is a number, or a [rows] tensor
        (float32; top_k: int32).  Returns the int32 tokens, or with ``logp`` also
        their float32 log-probabilities among the entries that the filters keep (numbers
        without a gradient)."""
        dtype = self._dtype("logits", logits)
        data, rows, vocab, stride = self._rows("logits", logits)
        if u is None:
            raise ValueError("u is needed")
        f32 = self._f32
        T, T_rows = self._setting("temperature", temperature, rows, f32)
        k, k_rows = self._setting("top_k", top_k, rows, self._i32)
        p, p_rows = self._setting("top_p", top_p, rows, f32)
        m, m_rows = self._setting("min_p", min_p, rows, f32)
        if not 0 <= k <= 0xFFFFFFFF:
            raise ValueError("top_k must be >= 0")
        token = self._empty(rows, dtype=self._i32, device=self.device)
        lp = self._empty(rows, dtype=f32, device=self.device) if logp else None
        args = rlsim_sample(dtype, data, rows, vocab, stride, self._vector("u", u, rows, f32), T, k, p, m,
                            T_rows, k_rows, p_rows, m_rows, token.data_ptr(), lp.data_ptr() if logp else None)
        if rows:                                  # an empty batch asks nothing of the device
            rlsim_head_sample(self.h, args)
        return (token, lp) if logp else token

    def distill(self, logits, teacher, index, temperature: float = 1.0, rest=None, weight=None, loss: bool = True, grad=True):
        """Distil rows of student ``logits`` [rows, vocab] from a teacher's top logits
        ``teacher`` [rows, k] at the entries ``index`` [rows, k] (int32 or int64; outside
        the row: an empty slot), optionally with ``rest`` [rows], the log of the sum of
        exp(t / temperature) over what it does not list.  Returns the float32 losses
        [rows] and the gradient of sum(weight * loss) in the logits' type; ``loss``
        or ``grad`` False leaves that one out.  ``grad`` may be a tensor to write to,
        the logits themselves among them; autograd takes that for any other write in place."""
        return self._distill(rlsim_head_distill, logits, teacher, index, temperature, rest, weight, loss, grad)

    def _distill(self, launch, logits, teacher, index, temperature, rest, weight, loss, grad):
        """distill, its marshalled call made by launch(handle, arguments)."""
        dtype = self._dtype("logits", logits)
        data, rows, vocab, stride = self._rows("logits", logits)
        t_dtype = self._dtype("teacher", teacher)
        t_data, _, k, t_stride = self._rows("teacher", teacher, rows)
        if index.dtype not in self._index:
            raise ValueError("index must be int32 or int64")
        i_data, _, _, i_stride = self._rows("index", index, rows, k)
        losses = self._empty(rows, dtype=self._f32, device=self.device) if loss else None
        out, g_data, g_stride = None, None, 0
        if grad is not False:
            out = self._empty((rows, vocab), dtype=logits.dtype, device=self.device) if grad is True else grad
            if out.dtype != logits.dtype:
                raise ValueError("grad must have the logits' type")
            g_data, _, _, g_stride = self._rows("grad", out, rows, vocab)
        args = rlsim_distill(dtype, data, rows, vocab, stride, t_dtype, t_data, t_stride,
                             self._index[index.dtype], i_data, i_stride, k, temperature,
                             self._vector("rest", rest, rows, self._f32), self._vector("weight", weight, rows, self._f32),
                             losses.data_ptr() if loss else None, g_data, g_stride)
        if rows:                                  # an empty batch asks nothing of the device
            launch(self.h, args)
        if out is not None and out is grad:
            self._written(out)                    # autograd cannot see a write through an address
        if loss and out is not None:
            return losses, out
        return losses if loss else out

    def distill_loss(self, logits, teacher, index, temperature: float = 1.0, rest=None):
        """The losses of ``distill`` [rows], differentiable with respect to ``logits``
        (the teacher is a constant).  Forward and backward are in order with the current
        stream, whichever the handle's is."""
        return _distill_function(self._torch).apply(self, logits, teacher, index, temperature, rest)

    def _launch_in_order(self, h, args):
        """Launch after what the current stream has been given, and before what it will be.
        Autograd makes, uses and frees tensors on the current stream inside its backward
        pass, where a caller can order nothing.  With both waits a tensor freed on the
        current stream is not written to again before the kernel is done with it."""
        current = self._torch.cuda.current_stream(self.device)
        elsewhere = current.cuda_stream != self._stream.cuda_stream
        if elsewhere:
            self._stream.wait_stream(current)
        rlsim_head_distill(h, args)
        if elsewhere:
            current.wait_stream(self._stream)


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
                return head._distill(head._launch_in_order, logits, teacher, index, temperature, rest, None, True, False)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, g):
                logits, teacher, index, *rest = ctx.saved_tensors
                out = ctx.head._distill(ctx.head._launch_in_order, logits, teacher, index, ctx.temperature,
                                        rest[0] if rest else None, g.contiguous(), False, True)
                return None, out, None, None, None, None

        _function = DistillLoss
    return _function
