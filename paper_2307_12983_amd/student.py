"""Thin ctypes binding over the operators of a student policy (declared in ``include/pql_student.h``).

Like ``binding``: argument marshalling only, every method of ``StudentContext`` forwards device pointers and
sizes to the C entry point of the same name.  Tensors are described once by the small classes below (they
hold the tensor, its C descriptor and what a call compares), so that a call made every step repeats little; it
still checks that what it is given belongs together, since the kernels would read and write out of range.
"""
from __future__ import annotations

import ctypes as C

from . import binding as B

PQL_F32, PQL_BF16 = 0, 1
PQL_MAX_TOP = 256
PQL_DELTA_MAX_DIM_K, PQL_DELTA_MAX_DIM_V = 128, 256

# every symbol include/pql_student.h declares
EXPORTS = ["pql_delta_step", "pql_delta_saved_bytes", "pql_delta_workspace_bytes", "pql_delta_forward",
           "pql_delta_backward", "pql_top_logits_workspace_bytes", "pql_top_logits", "pql_distill_workspace_bytes",
           "pql_distill_loss", "pql_distill_backward"]


class PqlSeq(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_b", C.c_int64), ("stride_t", C.c_int64), ("stride_h", C.c_int64)]


class PqlDeltaShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "steps", "heads_k", "heads_v", "dim_k", "dim_v", "dtype")] + \
               [("scale", C.c_float)]


class PqlDeltaInput(C.Structure):
    _fields_ = [(n, PqlSeq) for n in ("q", "k", "v", "log_decay", "beta")] + [("lengths", C.c_void_p), ("state", C.c_void_p)]


class PqlDeltaGrad(C.Structure):
    _fields_ = [(n, PqlSeq) for n in ("q", "k", "v", "log_decay", "beta")] + [("state", C.c_void_p)]


class PqlLogits(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_int64), ("stride", C.c_int64), ("vocab", C.c_int32), ("dtype", C.c_int32)]


class PqlTeacher(C.Structure):
    _fields_ = [("index", C.c_void_p), ("value", C.c_void_p), ("top", C.c_int32)]


_ready = None


def load_library() -> C.CDLL:
    """libpql.so with the prototypes of this module's entry points set."""
    global _ready
    if _ready is not None:
        return _ready
    lib = B.load_library()
    P, I32, I64, F = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    shape, logits = C.POINTER(PqlDeltaShape), C.POINTER(PqlLogits)
    given, grad = C.POINTER(PqlDeltaInput), C.POINTER(PqlDeltaGrad)
    sig = {
        "pql_delta_step": (I32, [P, shape, given, P, PqlSeq, P]),
        "pql_delta_saved_bytes": (I64, [shape]),
        "pql_delta_workspace_bytes": (I64, [shape, I32]),
        "pql_delta_forward": (I32, [P, shape, given, PqlSeq, P, P, P, P]),
        "pql_delta_backward": (I32, [P, shape, given, P, PqlSeq, P, grad, P, P]),
        "pql_top_logits_workspace_bytes": (I64, [logits, I32]),
        "pql_top_logits": (I32, [P, PqlLogits, I32, P, P, P, P]),
        "pql_distill_workspace_bytes": (I64, [logits]),
        "pql_distill_loss": (I32, [P, PqlLogits, PqlTeacher, F, P, P, P, PqlLogits, P, P]),
        "pql_distill_backward": (I32, [P, PqlLogits, PqlTeacher, F, P, P, PqlLogits, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _ready = lib
    return lib


_codes = {}
_f32 = _i32 = None                              # torch's types, found with the first tensor that is described


def _code(t):
    """PQL_F32, PQL_BF16, or None for any other type."""
    global _f32, _i32
    if not _codes:
        import torch
        _f32, _i32 = torch.float32, torch.int32
        _codes.update({torch.float32: PQL_F32, torch.bfloat16: PQL_BF16})
    return _codes.get(t.dtype)


def dtype_code(t) -> int:
    code = _code(t)
    if code is None:
        raise TypeError("tokens and logits are float32 or bfloat16, not %s" % t.dtype)
    return code


def workspace(nbytes: int, device="cuda"):
    """A device buffer of at least nbytes, 256-byte aligned (None for 0 bytes)."""
    if nbytes < 0:
        raise B.PqlError(nbytes, "workspace")
    if nbytes == 0:
        return None
    import torch
    t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    assert t.data_ptr() % 256 == 0
    return t


def _state(t, what: str, like):
    """The pointer of a contiguous float32 tensor of that shape; None stays None."""
    if t is None:
        return None
    if t.dtype is not _f32 or t.shape != like or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous float32 tensor of shape %s" % (what, like))
    return t.data_ptr()


def _values(t, what: str, count: int, dtype):
    """The pointer of a contiguous tensor of so many elements; None stays None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != count or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous tensor of %d elements of %s" % (what, count, dtype))
    return t.data_ptr()


class Sequence:
    """A token tensor [batch, steps, heads, dim] (or [batch, steps, heads] for gates) of any strides whose last
    dimension is contiguous."""

    def __init__(self, t):
        if t.dim() not in (3, 4):
            raise ValueError("token tensors have the dimensions batch, steps, heads and, gates apart, dim")
        if t.dim() == 4 and t.shape[3] > 1 and t.stride(3) != 1 and t.numel() > 0:
            raise ValueError("the last dimension of a token tensor must be contiguous")
        self.tensor = t
        self.key = (*t.shape, _code(t))
        self.c = PqlSeq(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))


def delta_shape(q, v, scale: float) -> PqlDeltaShape:
    """The shape of a call from its queries [batch, steps, heads_k, dim_k] and values [batch, steps, heads_v, dim_v]."""
    if q.dim() != 4 or v.dim() != 4 or q.shape[:2] != v.shape[:2] or q.dtype != v.dtype:
        raise ValueError("q and v: [batch, steps, heads, dim] of one type, batch and steps equal")
    return PqlDeltaShape(q.shape[0], q.shape[1], q.shape[2], v.shape[2], q.shape[3], v.shape[3], dtype_code(q), scale)


def _same(what, *pairs):
    for t, shape, dtype in pairs:
        if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
            raise ValueError("%s: shape %s of %s expected, got %s of %s" % (what, tuple(shape), dtype, tuple(t.shape), t.dtype))


class _Described:
    def __init__(self, struct, q, k, v, log_decay, beta, state, what):
        import torch
        n, t, hv, dv = v.shape
        _same(what, (k, q.shape, q.dtype), (v, (n, t, hv, dv), q.dtype), (log_decay, (n, t, hv), torch.float32),
              (beta, (n, t, hv), torch.float32))
        self.tensors = (q, k, v, log_decay, beta, state)
        self.shape = tuple(q.shape) + (hv, dv)
        self.key = (*self.shape, dtype_code(q))
        self.out_key, self.state_shape = (n, t, hv, dv, self.key[-1]), (n, hv, q.shape[3], dv)
        self.c = struct()
        for name, x in zip(("q", "k", "v", "log_decay", "beta"), self.tensors):
            setattr(self.c, name, Sequence(x).c)
        self.c.state = _state(state, what + ": state", self.state_shape)
        self.ref = C.byref(self.c)


class DeltaInput(_Described):
    """What the gated delta rule reads.  log_decay, beta: float32 [batch, steps, heads_v]; lengths: int32 [batch] or
    None; state: float32 [batch, heads_v, dim_k, dim_v] or None (zeros)."""

    def __init__(self, q, k, v, log_decay, beta, lengths=None, state=None):
        import torch
        super().__init__(PqlDeltaInput, q, k, v, log_decay, beta, state, "DeltaInput")
        if lengths is not None and (lengths.dtype != torch.int32 or tuple(lengths.shape) != (q.shape[0],) or not lengths.is_contiguous()):
            raise ValueError("DeltaInput: lengths are a contiguous int32 tensor [batch]")
        self.lengths = lengths
        self.c.lengths = None if lengths is None else lengths.data_ptr()


class DeltaGrad(_Described):
    """Where the gradients go; the shapes of the inputs, state may be None."""

    def __init__(self, q, k, v, log_decay, beta, state=None):
        super().__init__(PqlDeltaGrad, q, k, v, log_decay, beta, state, "DeltaGrad")


class Logits:
    """Rows of logits [rows, vocab], contiguous within a row."""

    def __init__(self, t):
        if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
            raise ValueError("logits: [rows, vocab], contiguous within a row")
        self.tensor, self.rows = t, t.shape[0]
        stride = t.stride(0) if t.shape[0] > 1 else t.shape[1]
        self.c = PqlLogits(t.data_ptr(), t.shape[0], stride, t.shape[1], dtype_code(t))


class Teacher:
    """A teacher's lists: index int32 [rows, top] (outside the vocabulary: no entry), value float32 [rows, top]."""

    def __init__(self, index, value):
        import torch
        if index.dim() != 2 or index.shape != value.shape or index.dtype != torch.int32 or value.dtype != torch.float32 \
                or not index.is_contiguous() or not value.is_contiguous():
            raise ValueError("lists are contiguous int32 and float32 tensors [rows, top]")
        self.index, self.value, self.rows = index, value, index.shape[0]
        self.c = PqlTeacher(index.data_ptr(), value.data_ptr(), index.shape[1])


NO_GRAD = PqlLogits(None, 0, 0, 0, 0)


class StudentContext(B.Context):
    """A context whose methods are the student's entry points beside those of ``binding.Context``.  Without a
    configuration it serves the student's calls alone."""

    def __init__(self, cfg: B.PqlConfig = None):
        load_library()
        super().__init__(cfg if cfg is not None else B.make_config(1, 1, 1, 1, 1, 1.0, (1,), 1, 0))

    # ---- host queries
    def delta_saved_bytes(self, shape: PqlDeltaShape) -> int:
        return self.lib.pql_delta_saved_bytes(C.byref(shape))

    def delta_workspace_bytes(self, shape: PqlDeltaShape, backward: bool) -> int:
        return self.lib.pql_delta_workspace_bytes(C.byref(shape), int(backward))

    def top_logits_workspace_bytes(self, logits: Logits, top: int) -> int:
        return self.lib.pql_top_logits_workspace_bytes(C.byref(logits.c), top)

    def distill_workspace_bytes(self, logits: Logits) -> int:
        return self.lib.pql_distill_workspace_bytes(C.byref(logits.c))

    # ---- device calls
    @staticmethod
    def _fits(s, given, out):
        if given.key != (s.batch, s.steps, s.heads_k, s.dim_k, s.heads_v, s.dim_v, s.dtype) or out.key != given.out_key:
            raise ValueError("tensors and shape of the call do not agree")

    @staticmethod
    def _state(given, t, what):
        return given.c.state if t is given.tensors[5] else _state(t, what, given.state_shape)

    def pql_delta_step(self, shape, given: DeltaInput, state_out, out: Sequence, stream=None):
        self._fits(shape, given, out)
        state_out = self._state(given, state_out, "state_out")
        self._check(self.lib.pql_delta_step(self.h, C.byref(shape), given.ref, state_out, out.c, B._stream(stream)))

    def pql_delta_forward(self, shape, given: DeltaInput, out: Sequence, state_out, saved, workspace, stream=None):
        self._fits(shape, given, out)
        state_out = self._state(given, state_out, "state_out")
        self._check(self.lib.pql_delta_forward(self.h, C.byref(shape), given.ref, out.c, state_out, B._ptr(saved),
                                               B._ptr(workspace), B._stream(stream)))

    def pql_delta_backward(self, shape, given: DeltaInput, saved, out_grad: Sequence, state_out_grad, grads: DeltaGrad,
                           workspace, stream=None):
        self._fits(shape, given, out_grad)
        self._fits(shape, grads, out_grad)
        state_out_grad = self._state(given, state_out_grad, "state_out_grad")
        self._check(self.lib.pql_delta_backward(self.h, C.byref(shape), given.ref, B._ptr(saved), out_grad.c,
                                                state_out_grad, grads.ref, B._ptr(workspace), B._stream(stream)))

    def pql_top_logits(self, logits: Logits, top, index_out, value_out, workspace, stream=None):
        n = logits.rows * top
        index_out, value_out = _values(index_out, "index_out", n, _i32), _values(value_out, "value_out", n, _f32)
        self._check(self.lib.pql_top_logits(self.h, logits.c, top, index_out, value_out, B._ptr(workspace), B._stream(stream)))

    @staticmethod
    def _rows(logits, teacher):
        if teacher.rows != logits.rows:
            raise ValueError("the teacher's lists are of %d rows, the logits of %d" % (teacher.rows, logits.rows))
        return logits.rows

    def pql_distill_loss(self, logits: Logits, teacher: Teacher, temperature, row_weight, loss_out, lse_out, grad,
                         workspace, stream=None):
        n = self._rows(logits, teacher)
        self._check(self.lib.pql_distill_loss(self.h, logits.c, teacher.c, temperature, _values(row_weight, "row_weight", n, _f32),
                                              _values(loss_out, "loss_out", n, _f32), _values(lse_out, "lse_out", n, _f32),
                                              NO_GRAD if grad is None else grad.c, B._ptr(workspace), B._stream(stream)))

    def pql_distill_backward(self, logits: Logits, teacher: Teacher, temperature, lse, loss_grad, grad: Logits, stream=None):
        n = self._rows(logits, teacher)
        self._check(self.lib.pql_distill_backward(self.h, logits.c, teacher.c, temperature, _values(lse, "lse", n, _f32),
                                                  _values(loss_grad, "loss_grad", n, _f32), grad.c, B._stream(stream)))
