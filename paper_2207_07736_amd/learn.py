"""Thin Python binding of the learner's operators (rlsim_learner_* of include/rlsim.h):
argument marshalling only.

``Learner`` has the gated recurrence over recorded rows, the cross entropy of an output
layer and clipping by the global norm.  torch is used for device memory, and so that
``Learner.recur`` and ``Learner.cross_entropy_loss`` can take part in its backward pass.
"""
from __future__ import annotations

import array
import ctypes

from .rlsim import RLSIM_BF16, RLSIM_F16, RLSIM_F32, RLSIM_OK, RlsimError, lib

RLSIM_SCAN_MARK = 16

_u32, _u64, _ptr, _int = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_int


class rlsim_scan(ctypes.Structure):
    _fields_ = [("dtype", _int), ("T", _u32), ("n", _u32), ("channels", _u32), ("x", _ptr), ("gate", _ptr),
                ("x_step", _u64), ("x_seq", _u64), ("gate_step", _u64), ("gate_seq", _u64), ("state", _ptr),
                ("done", _ptr), ("marks", _ptr), ("y", _ptr), ("y_step", _u64), ("y_seq", _u64), ("last", _ptr)]


class rlsim_scan_grad(ctypes.Structure):
    _fields_ = [("dy", _ptr), ("dy_step", _u64), ("dy_seq", _u64), ("dlast", _ptr), ("dx", _ptr), ("dgate", _ptr),
                ("dx_step", _u64), ("dx_seq", _u64), ("dgate_step", _u64), ("dgate_seq", _u64), ("dstate", _ptr)]


class rlsim_xent(ctypes.Structure):
    _fields_ = [("dtype", _int), ("rows", _u32), ("dim", _u32), ("vocab", _u32), ("hidden", _ptr),
                ("hidden_stride", _u64), ("matrix", _ptr), ("matrix_stride", _u64), ("target_bytes", _int),
                ("target", _ptr), ("weight", _ptr), ("loss", _ptr), ("stats", _ptr), ("dhidden", _ptr),
                ("dhidden_stride", _u64), ("dmatrix", _ptr), ("dmatrix_stride", _u64)]


class rlsim_tensor(ctypes.Structure):
    _fields_ = [("data", _ptr), ("out", _ptr), ("elements", _u64), ("dtype", _int), ("out_dtype", _int)]


lib.rlsim_learner_create.argtypes = [_u32, _u32, _u32, _ptr, ctypes.POINTER(_ptr)]
lib.rlsim_learner_scan.argtypes = [_ptr, ctypes.POINTER(rlsim_scan)]
lib.rlsim_learner_scan_grad.argtypes = [_ptr, ctypes.POINTER(rlsim_scan), ctypes.POINTER(rlsim_scan_grad)]
lib.rlsim_learner_xent.argtypes = [_ptr, ctypes.POINTER(rlsim_xent)]
lib.rlsim_learner_clip.argtypes = [_ptr, _ptr, _u32, ctypes.c_double, _ptr]
lib.rlsim_learner_destroy.argtypes = [_ptr]
for _name in ("create", "scan", "scan_grad", "xent", "clip", "destroy"):
    getattr(lib, "rlsim_learner_" + _name).restype = _int
lib.rlsim_learner_last_error.argtypes = [_ptr]
lib.rlsim_learner_last_error.restype = ctypes.c_char_p


def _check_learner(rc: int, h) -> None:
    if rc != RLSIM_OK:
        msg = lib.rlsim_learner_last_error(h)
        raise RlsimError(rc, msg.decode() if msg else "rlsim error")


def rlsim_learner_last_error(h=None) -> str:
    return lib.rlsim_learner_last_error(h).decode()


def rlsim_learner_create(max_rows: int = 0, max_dim: int = 0, max_vocab: int = 0, stream=None) -> ctypes.c_void_p:
    """A learner's handle; ``stream`` is a torch.cuda.Stream, a raw hipStream_t int, or
    None for the default stream."""
    if stream is not None:
        stream = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    h = ctypes.c_void_p()
    _check_learner(lib.rlsim_learner_create(int(max_rows), int(max_dim), int(max_vocab), stream, ctypes.byref(h)), None)
    return h


def rlsim_learner_scan(h, args: rlsim_scan) -> None:
    rc = lib.rlsim_learner_scan(h, ctypes.byref(args))
    if rc:
        _check_learner(rc, h)


def rlsim_learner_scan_grad(h, args: rlsim_scan, grad: rlsim_scan_grad) -> None:
    rc = lib.rlsim_learner_scan_grad(h, ctypes.byref(args), ctypes.byref(grad))
    if rc:
        _check_learner(rc, h)


def rlsim_learner_xent(h, args: rlsim_xent) -> None:
    rc = lib.rlsim_learner_xent(h, ctypes.byref(args))
    if rc:
        _check_learner(rc, h)


def rlsim_learner_clip(h, tensors, count: int, max_norm: float, norm) -> None:
    """``tensors``: a ctypes array of rlsim_tensor (or its address); ``norm``: a device
    address."""
    rc = lib.rlsim_learner_clip(h, tensors, count, max_norm, norm)
    if rc:
        _check_learner(rc, h)


def rlsim_learner_destroy(h) -> None:
    if h:
        _check_learner(lib.rlsim_learner_destroy(h), None)


class Learner:
    """Owning wrapper of one learner's handle.  ``max_rows``, ``max_dim`` and
    ``max_vocab`` bound its ``cross_entropy`` calls (all 0: none are made); ``scan`` and
    ``clip`` take any size.  Tensors are on the device the handle was created on, and are
    used on the handle's stream: work that makes or frees them elsewhere has to be ordered
    with it (``recur`` and ``cross_entropy_loss`` order themselves).  That holds for the
    returned tensors too, which torch allocates for its current stream.  All calls of a
    handle, and all replays of graphs that captured some, have to be ordered with one
    another: graphs that may run at the same time need a Learner each, and none is
    replayed once its Learner is closed.  ``recur`` and ``cross_entropy_loss`` are not
    captured (torch's own bookkeeping of leaves does not allow it everywhere): a captured
    step calls ``scan``, ``scan_grad`` and ``cross_entropy``."""

    def __init__(self, max_rows: int = 0, max_dim: int = 0, max_vocab: int = 0, stream=None):
        import torch
        self.h = None
        self._dtypes = {torch.float32: RLSIM_F32, torch.bfloat16: RLSIM_BF16, torch.float16: RLSIM_F16}
        self._types = {t: d | d << 32 for t, d in self._dtypes.items()}          # both types of an rlsim_tensor
        self._target = {torch.uint8: 1, torch.int32: 4, torch.int64: 8}
        self._torch, self._empty, self._empty_like = torch, torch.empty, torch.empty_like
        self._written = torch.autograd.graph.increment_version
        self._f32, self._strided = torch.float32, torch.strided
        self._done = (torch.uint8, torch.bool)
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._ordinal = self.device.index
        self.max_rows, self.max_dim, self.max_vocab = int(max_rows), int(max_dim), int(max_vocab)
        if stream is None or not hasattr(stream, "cuda_stream"):
            stream = (torch.cuda.ExternalStream(int(stream), device=self.device) if stream
                      else torch.cuda.default_stream(self.device))
        self._stream = stream
        self.h = rlsim_learner_create(max_rows, max_dim, max_vocab, stream)

    def close(self):
        if self.h:
            h, self.h = self.h, None
            rlsim_learner_destroy(h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _dtype(self, name, t):
        try:
            return self._dtypes[t.dtype]
        except KeyError:
            raise ValueError(f"{name} must be float32, bfloat16 or float16") from None

    # ---- the gated recurrence ------------------------------------------------------

    def _rows(self, name, t, shape, dtype):
        """Address and (step, sequence) strides of a [T, n, channels] tensor whose
        channels are consecutive elements."""
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self._ordinal:
            raise ValueError(f"{name} must be {dtype}, {list(shape)}, on {self.device}")
        step, seq, one = t.stride()
        if one != 1 and shape[2] > 1:
            raise ValueError(f"{name} must hold each row's channels in consecutive elements")
        return t.data_ptr(), step, seq

    def _plain(self, name, t, shape, dtype=None):
        """The address of a contiguous tensor, None for None."""
        if t is None:
            return None
        dtype = dtype or self._f32
        if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != self._ordinal:
            raise ValueError(f"{name} must be {dtype}, {list(shape)}, contiguous, on {self.device}")
        return t.data_ptr()

    def _ends(self, done, T, n):
        if done is None:
            return None
        if done.dtype not in self._done:
            raise ValueError("done must be uint8 or bool")
        return self._plain("done", done, (T, n), done.dtype)

    def _scan_args(self, x, gate, state, done, marks, y, y_step, y_seq, last):
        shape, kind = x.shape, x.dtype
        T, n, channels = shape
        x_at, x_step, x_seq = self._rows("x", x, shape, kind)
        g_at, g_step, g_seq = self._rows("gate", gate, shape, kind)
        return rlsim_scan(self._dtypes[kind], T, n, channels, x_at, g_at, x_step, x_seq, g_step, g_seq,
                          None if state is None else self._plain("state", state, (n, channels)),
                          None if done is None else self._ends(done, T, n), marks, y, y_step, y_seq, last)

    def _scan_shape(self, x):
        if x.dtype not in self._dtypes:
            raise ValueError("x must be float32, bfloat16 or float16")
        if x.dim() != 3:
            raise ValueError("x must be 3-d, [T, n, channels]")
        return x.shape

    def _like(self, x):
        """A new tensor of x's shape and order of its first two dimensions."""
        if x.is_contiguous():
            return self._empty_like(x)
        T, n, channels = x.shape
        if n > 1 and T > 1 and x.stride(1) > x.stride(0):
            return self._empty((n, T, channels), dtype=x.dtype, device=self.device).transpose(0, 1)
        return self._empty((T, n, channels), dtype=x.dtype, device=self.device)

    def scan(self, x, gate, state=None, done=None, marks: bool = False, last=None):
        """The gated recurrence h_t = a_t h'_{t-1} + (1 - a_t) x_t, a_t = sigmoid(gate_t),
        over ``x`` and ``gate`` [T, n, channels] (channels in consecutive elements; T and n
        in either order in memory), from ``state`` [n, channels] (float32; None: 0).  Where
        ``done`` [T, n] (uint8 or bool) is not 0 an episode ends with the step: h' is 0
        there, h elsewhere.  Returns the h_t in x's type and h'_{T-1} in float32, written to
        ``last`` if given (``state`` itself among others); with ``marks`` also what
        ``scan_grad`` needs.  T = 1 is a step of acting."""
        return self._scan(rlsim_learner_scan, x, gate, state, done, marks, last)

    def _scan(self, launch, x, gate, state, done, marks, last):
        T, n, channels = self._scan_shape(x)
        y = self._like(x)
        y_step, y_seq, _ = y.stride()
        given = last is not None
        if given:
            at = self._plain("last", last, (n, channels))
        else:
            last = (self._empty_like(state) if state is not None and state.is_contiguous()
                    else self._empty((n, channels), dtype=self._f32, device=self.device))
            at = last.data_ptr()
        kept = self._empty((-(-T // RLSIM_SCAN_MARK), n, channels), dtype=self._f32, device=self.device) if marks else None
        args = self._scan_args(x, gate, state, done, kept.data_ptr() if marks else None, y.data_ptr(), y_step, y_seq, at)
        if T and n and channels:
            launch(self.h, args)
        elif n and channels:                      # no steps: the state as it was
            if state is None:
                last.zero_()
            elif last is not state:
                last.copy_(state)
        if given:
            self._written(last)                   # autograd cannot see a write through an address
        return (y, last, kept) if marks else (y, last)

    def scan_grad(self, x, gate, marks, dy=None, done=None, dlast=None):
        """The gradients of ``scan``'s x, gate and state (float32) from those of its h_t
        (``dy``; None: 0) and of its last state (``dlast`` [n, channels], float32; None: 0).
        ``marks`` are what ``scan`` returned for the same x, gate, state and done."""
        return self._scan_grad(rlsim_learner_scan_grad, x, gate, marks, dy, done, dlast)

    def _scan_grad(self, launch, x, gate, marks, dy, done, dlast):
        T, n, channels = shape = self._scan_shape(x)
        if marks is None:
            raise ValueError("marks are needed")
        args = self._scan_args(x, gate, None, done, self._plain("marks", marks, (-(-T // RLSIM_SCAN_MARK), n, channels)),
                               None, 0, 0, None)
        dx, dgate = self._like(x), self._like(x)
        dstate = self._empty((n, channels), dtype=self._f32, device=self.device)
        step, seq, _ = dx.stride()
        g = rlsim_scan_grad(*((None, 0, 0) if dy is None else self._rows("dy", dy, shape, x.dtype)),
                            self._plain("dlast", dlast, (n, channels)), dx.data_ptr(), dgate.data_ptr(), step, seq, step, seq,
                            dstate.data_ptr())
        if T and n and channels:
            launch(self.h, args, g)
        elif n and channels:
            dstate.zero_() if dlast is None else dstate.copy_(dlast)
        return dx, dgate, dstate

    def recur(self, x, gate, state=None, done=None):
        """``scan`` as (h, last state), differentiable with respect to ``x``, ``gate`` and
        ``state``.  Forward and backward are in order with the current stream, whichever
        the handle's is."""
        return _functions(self._torch)[0].apply(self, x, gate, state, done)

    # ---- the output layer's cross entropy ------------------------------------------

    def _matrix(self, name, t, rows, width, dtype):
        """Address and row stride of a [rows, width] tensor of whole rows."""
        if t.dtype != dtype or t.shape != (rows, width) or t.get_device() != self._ordinal:
            raise ValueError(f"{name} must be {dtype}, [{rows}, {width}], on {self.device}")
        if t.is_contiguous():
            return t.data_ptr(), width
        stride, step = t.stride()
        stride = stride if rows > 1 else width
        if (width > 1 and step != 1) or stride < width:
            raise ValueError(f"{name} must hold each row in consecutive elements, rows apart")
        return t.data_ptr(), stride

    def cross_entropy(self, hidden, matrix, target, weight=None, loss: bool = True, grad=True, stats=None):
        """The cross entropy of the output layer z = hidden matrix^T: ``hidden``
        [rows, dim], ``matrix`` [vocab, dim] of the same type, ``target`` [rows] (uint8,
        int32 or int64; outside the vocabulary: the row counts for nothing).  Returns the
        float32 losses [rows] and the gradients of sum(weight * loss) with respect to
        ``hidden`` and ``matrix``, ``weight`` [rows] in float32 (None: 1).  ``loss`` False
        leaves the losses out and takes ``stats``; ``grad`` False leaves out both
        gradients, "hidden" or "matrix" is that one alone.  ``stats`` [rows, 3] (float32)
        receives each row's largest logit and the sums of exp(z - largest) without and of
        its target, which a call for gradients alone takes back."""
        return self._cross_entropy(rlsim_learner_xent, hidden, matrix, target, weight, loss, grad, stats)

    def _cross_entropy(self, launch, hidden, matrix, target, weight, loss, grad, stats):
        if grad is not True and grad is not False and grad != "hidden" and grad != "matrix":
            raise ValueError('grad must be True, False, "hidden" or "matrix"')
        if not loss and grad is False:
            raise ValueError("neither loss nor grad is wanted")
        if not loss and stats is None:
            raise ValueError("gradients alone need stats")
        dtype = self._dtype("hidden", hidden)
        if hidden.dim() != 2 or matrix.dim() != 2:
            raise ValueError("hidden must be [rows, dim], matrix [vocab, dim]")
        rows, dim = hidden.shape
        vocab = matrix.shape[0]
        if target.dtype not in self._target:
            raise ValueError("target must be uint8, int32 or int64")
        h_at, h_stride = self._matrix("hidden", hidden, rows, dim, hidden.dtype)
        m_at, m_stride = self._matrix("matrix", matrix, vocab, dim, hidden.dtype)
        target_at = self._plain("target", target, (rows,), target.dtype)
        weight_at, stats_at = self._plain("weight", weight, (rows,)), self._plain("stats", stats, (rows, 3))
        out, loss_at, dh_at, dm_at = [], None, None, None
        if loss:
            losses = self._empty(rows, dtype=self._f32, device=self.device)
            loss_at = losses.data_ptr()
            out.append(losses)
        if grad is True or grad == "hidden":
            dhidden = self._empty_like(hidden) if hidden.is_contiguous() else self._empty((rows, dim), dtype=hidden.dtype, device=self.device)
            dh_at = dhidden.data_ptr()
            out.append(dhidden)
        if grad is True or grad == "matrix":
            dmatrix = self._empty_like(matrix) if matrix.is_contiguous() else self._empty((vocab, dim), dtype=hidden.dtype, device=self.device)
            dm_at = dmatrix.data_ptr()
            out.append(dmatrix)
        args = rlsim_xent(dtype, rows, dim, vocab, h_at, h_stride, m_at, m_stride, self._target[target.dtype], target_at,
                          weight_at, loss_at, stats_at, dh_at, dim, dm_at, dim)
        if rows:
            launch(self.h, args)
        elif dm_at is not None:                   # an empty batch teaches nothing
            out[-1].zero_()
        if loss and stats is not None:
            self._written(stats)
        return tuple(out) if len(out) > 1 else out[0]

    def cross_entropy_loss(self, hidden, matrix, target):
        """The losses of ``cross_entropy`` [rows], differentiable with respect to
        ``hidden`` and ``matrix``.  Forward and backward are in order with the current
        stream, whichever the handle's is."""
        return _functions(self._torch)[1].apply(self, hidden, matrix, target)

    # ---- clipping ------------------------------------------------------------------

    def _dense(self, name, t):
        """Whether t's elements lie side by side, in whatever order."""
        if t.layout is not self._strided or t.get_device() != self._ordinal:
            raise ValueError(f"{name} must be a dense tensor on {self.device}")
        if t.is_contiguous():
            return
        expected = 1
        for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
            if stride != expected:
                raise ValueError(f"{name} must hold its elements side by side")
            expected *= size

    def clip(self, tensors, max_norm: float, out=None):
        """Scale ``tensors`` (float32, bfloat16 or float16; None entries are skipped) in
        place by max_norm / norm where their global norm is finite and above ``max_norm``.
        ``out``: tensors to write to instead, each with its tensor's elements in the same
        order in memory, of any of the types.  Returns the norm before, a float32 number on the
        device."""
        if not max_norm > 0:
            raise ValueError("max_norm must be > 0")
        tensors = list(tensors)
        if out is not None:
            out = list(out)
            if len(out) != len(tensors):
                raise ValueError("out must have a tensor for each")
            pairs = [(t, o) for t, o in zip(tensors, out) if t is not None]
        else:
            pairs = [(t, t) for t in tensors if t is not None]
        words, types, ordinal, here = [], self._types, self._ordinal, self._dense
        add = words.extend
        for t, o in pairs:
            kind = types.get(t.dtype)
            if kind is None:
                raise ValueError("tensors must be float32, bfloat16 or float16")
            if t.get_device() != ordinal or not t.is_contiguous():
                here("tensors", t)
            if o is t:
                add((t.data_ptr(), 0, t.numel(), kind))
                continue
            other = types.get(o.dtype) if o is not None else None
            if other is None:
                raise ValueError("out must be float32, bfloat16 or float16 tensors")
            n = t.numel()
            if o.get_device() != ordinal or not o.is_contiguous() or not t.is_contiguous():
                here("out", o)
                if o.shape != t.shape or o.stride() != t.stride():
                    raise ValueError("out must have its tensor's elements in the same order in memory")
            if o.numel() != n:
                raise ValueError("out must have as many elements as its tensor")
            add((t.data_ptr(), o.data_ptr(), n, kind & 0xFFFFFFFF | other & 0xFFFFFFFF00000000))
        table = array.array("Q", words)           # rows of an rlsim_tensor
        norm = self._empty((), dtype=self._f32, device=self.device)
        rlsim_learner_clip(self.h, table.buffer_info()[0], len(pairs), float(max_norm), norm.data_ptr())
        if pairs and (max_norm < float("inf") or out is not None):
            self._written([o for _, o in pairs])  # autograd cannot see a write through an address
        return norm

    def _in_order(self, launch, *args):
        """Launch after what the current stream has been given, and before what it will be.
        Autograd makes, uses and frees tensors on the current stream inside its backward
        pass, where a caller can order nothing."""
        current = self._torch.cuda.current_stream(self.device)
        elsewhere = current.cuda_stream != self._stream.cuda_stream
        if elsewhere:
            self._stream.wait_stream(current)
        launch(*args)
        if elsewhere:
            current.wait_stream(self._stream)

    def _not_captured(self, name):
        if self._torch.cuda.is_current_stream_capturing():
            raise RuntimeError(f"{name} is not captured: capture scan, scan_grad and cross_entropy")


_made = None


def _functions(torch):
    """The autograd functions behind Learner.recur and Learner.cross_entropy_loss, made
    on first use."""
    global _made
    if _made is not None:
        return _made

    class Recur(torch.autograd.Function):
        @staticmethod
        def forward(ctx, learner, x, gate, state, done):
            learner._not_captured("recur")
            ctx.learner, ctx.has = learner, (state is not None, done is not None)
            launch = lambda h, a: learner._in_order(rlsim_learner_scan, h, a)  # noqa: E731
            y, last, marks = learner._scan(launch, x, gate, state, done, True, None)
            ctx.save_for_backward(x, gate, marks, *(() if done is None else (done,)))
            ctx.set_materialize_grads(False)
            return y, last

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy, dlast):
            learner = ctx.learner
            learner._not_captured("recur")
            x, gate, marks, *done = ctx.saved_tensors
            if dy is not None and (dy.stride(2) != 1 and dy.shape[2] > 1):
                dy = dy.contiguous()
            launch = lambda h, a, g: learner._in_order(rlsim_learner_scan_grad, h, a, g)  # noqa: E731
            dx, dgate, dstate = learner._scan_grad(launch, x, gate, marks, dy, done[0] if done else None,
                                                   None if dlast is None else dlast.contiguous())
            return None, dx, dgate, dstate if ctx.has[0] else None, None

    class CrossEntropyLoss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, learner, hidden, matrix, target):
            learner._not_captured("cross_entropy_loss")
            ctx.learner = learner
            stats = torch.empty((hidden.shape[0], 3), dtype=torch.float32, device=learner.device)
            launch = lambda h, a: learner._in_order(rlsim_learner_xent, h, a)  # noqa: E731
            losses = learner._cross_entropy(launch, hidden, matrix, target, None, True, False, stats)
            ctx.save_for_backward(hidden, matrix, target, stats)
            return losses

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, g):
            learner = ctx.learner
            learner._not_captured("cross_entropy_loss")
            hidden, matrix, target, stats = ctx.saved_tensors
            wants = ctx.needs_input_grad[1], ctx.needs_input_grad[2]
            grad = True if all(wants) else "hidden" if wants[0] else "matrix"
            launch = lambda h, a: learner._in_order(rlsim_learner_xent, h, a)  # noqa: E731
            out = learner._cross_entropy(launch, hidden, matrix, target, g.contiguous(), False, grad, stats)
            if grad is True:
                return None, out[0], out[1], None
            return (None, out, None, None) if wants[0] else (None, None, out, None)

    _made = Recur, CrossEntropyLoss
    return _made
