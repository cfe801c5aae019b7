"""Thin ctypes binding over the operators around a student's memory (declared in ``include/pql_block.h``).

Like ``student``: argument marshalling only, every method of ``BlockContext`` forwards device pointers and sizes to the
C entry point of the same name.  Tensors are described once by the small classes below; a call checks that what it is
given belongs together, since the kernels would read and write out of range.
"""
from __future__ import annotations

import ctypes as C

from . import binding as B
from . import student as S

PQL_F32, PQL_BF16 = S.PQL_F32, S.PQL_BF16
ACTIVATIONS = {"none": 0, "sigmoid": 1, "silu": 2, "gelu": 3, "relu": 4}
PQL_RESIDUAL_MAX_DIM, PQL_RESIDUAL_MAX_GROUPS, PQL_FFN_MAX_DIM = 8192, 256, 65536
FFN_FORWARD, FFN_BACKWARD, FFN_BACKWARD_ALONE = 0, 1, 2
workspace = S.workspace

# every symbol include/pql_block.h declares
EXPORTS = ["pql_embed_forward", "pql_embed_workspace_bytes", "pql_embed_backward", "pql_residual_forward",
           "pql_residual_workspace_bytes", "pql_residual_backward", "pql_ffn_saved_bytes", "pql_ffn_workspace_bytes",
           "pql_ffn_forward", "pql_ffn_backward"]


class PqlRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64)]


class PqlEmbedShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "steps", "per_row", "vocab", "dim", "dtype")] + [("scale", C.c_float)]


class PqlResidualShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "steps", "dim", "groups", "dtype", "gate_cols", "gate_act")] + \
               [(n, C.c_float) for n in ("eps_post", "eps_pre", "scale_x", "scale_y")]


class PqlResidualInput(C.Structure):
    _fields_ = [(n, PqlRows) for n in ("x", "y", "gate")] + [(n, C.c_void_p) for n in ("post", "pre", "lengths")]


class PqlResidualGrad(C.Structure):
    _fields_ = [(n, PqlRows) for n in ("x", "y", "gate")] + [(n, C.c_void_p) for n in ("post", "pre")]


class PqlFfnShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "steps", "dim", "hidden", "dtype", "act")]


class PqlFfnInput(C.Structure):
    _fields_ = [(n, PqlRows) for n in ("x", "gate", "up", "down")] + [("lengths", C.c_void_p)]


class PqlFfnGrad(C.Structure):
    _fields_ = [(n, PqlRows) for n in ("x", "gate", "up", "down")]


_ready = None


def load_library() -> C.CDLL:
    """libpql.so with the prototypes of this module's entry points set."""
    global _ready
    if _ready is not None:
        return _ready
    lib = S.load_library()
    P, I32, I64 = C.c_void_p, C.c_int32, C.c_int64
    rows = C.POINTER(PqlRows)
    embed, residual, ffn = C.POINTER(PqlEmbedShape), C.POINTER(PqlResidualShape), C.POINTER(PqlFfnShape)
    r_in, r_grad, f_in, f_grad = (C.POINTER(x) for x in (PqlResidualInput, PqlResidualGrad, PqlFfnInput, PqlFfnGrad))
    sig = {
        "pql_embed_forward": (I32, [P, embed, P, P, rows, rows, P]),
        "pql_embed_workspace_bytes": (I64, [embed]),
        "pql_embed_backward": (I32, [P, embed, P, P, rows, rows, P, P]),
        "pql_residual_forward": (I32, [P, residual, r_in, rows, rows, P]),
        "pql_residual_workspace_bytes": (I64, [residual]),
        "pql_residual_backward": (I32, [P, residual, r_in, rows, rows, r_grad, P, P]),
        "pql_ffn_saved_bytes": (I64, [ffn]),
        "pql_ffn_workspace_bytes": (I64, [ffn, I32]),
        "pql_ffn_forward": (I32, [P, ffn, f_in, rows, P, P, P]),
        "pql_ffn_backward": (I32, [P, ffn, f_in, P, rows, f_grad, P, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _ready = lib
    return lib


class Rows:
    """A matrix [rows, cols] or token tensor [batch, steps, cols] whose rows are contiguous and equally far apart."""

    def __init__(self, t):
        if t.dim() not in (2, 3):
            raise ValueError("rows are tensors [rows, cols] or [batch, steps, cols]")
        cols = t.shape[-1]
        if cols > 1 and t.stride(-1) != 1 and t.numel() > 0:
            raise ValueError("the last dimension of rows must be contiguous")
        n, stride = (t.shape[0], t.stride(0)) if t.dim() == 2 or t.shape[1] == 1 else (t.shape[0] * t.shape[1], t.stride(1))
        if t.dim() == 3 and t.shape[0] > 1 and t.shape[1] > 1 and t.stride(0) != t.shape[1] * stride and t.numel() > 0:
            raise ValueError("the rows of a token tensor must be equally far apart")
        self.tensor, self.dev = t, t.get_device()
        self.key = (n, cols, S.dtype_code(t))
        self.c = PqlRows(t.data_ptr(), stride if n > 1 else cols)
        self.ref = C.byref(self.c)


def _one_device(what, *tensors):
    devices = {t.get_device() for t in tensors if t is not None}
    if len(devices) > 1:
        raise ValueError("%s: tensors of different devices" % what)
    return devices.pop() if devices else None


def _stream(stream, *devices):
    """The stream's handle; what a call is given has to lie on its device (the current one's stream, if it is None)."""
    if stream is None:                          # its handle alone: torch.cuda.current_stream() takes 2.7 us of a call of 8
        import torch
        here = torch.cuda.current_device()
        handle = torch._C._cuda_getCurrentRawStream(here) or None
    else:
        here, handle = getattr(stream, "device_index", None), B._stream(stream)
    for d in devices:
        if d is not None and (d < 0 or here is not None and d != here):
            raise ValueError("tensors of another device than the stream's")
    return handle


def _dev(*tensors):
    return [t.get_device() for t in tensors if t is not None]


NONE = PqlRows(None, 0)
_NO_ROWS = C.byref(NONE)


def _ref(rows, key, what):
    """The descriptor of rows that have to be like key; None stays none."""
    if rows is None:
        return _NO_ROWS
    if rows.key != key:
        raise ValueError("%s: %d rows of %d (type %d) expected, got %d rows of %d (type %d)" % ((what,) + key + rows.key))
    return rows.ref


def _rows(t, key, what):
    if t is None:
        return NONE
    r = Rows(t)
    _ref(r, key, what)
    return r.c


def _floats(t, count, what):
    import torch
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != count or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous float32 tensor of %d elements" % (what, count))
    return t.data_ptr()


def _ints(t, count, what):
    import torch
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.numel() != count or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous int32 tensor of %d elements" % (what, count))
    return t.data_ptr()


def _space(t, size, what):
    """The pointer of memory of at least so many bytes; None stays None."""
    if t is None:
        return None
    if t.numel() * t.element_size() < size or not t.is_contiguous():
        raise ValueError("%s: expected at least %d contiguous bytes, got %d" % (what, size, t.nbytes))
    return t.data_ptr()


def embed_shape(tokens, table, scale: float) -> PqlEmbedShape:
    """The shape of a call from its tokens [batch, steps, per_row] and its table [vocab, dim]."""
    if tokens.dim() != 3 or table.dim() != 2:
        raise ValueError("tokens: [batch, steps, per_row]; table: [vocab, dim]")
    return PqlEmbedShape(*tokens.shape, *table.shape, S.dtype_code(table), scale)


def residual_shape(batch, steps, dim, dtype, groups=1, gate_cols=0, gate_act="none", eps_post=0.0, eps_pre=0.0, scale_x=1.0,
                   scale_y=1.0) -> PqlResidualShape:
    """dtype: torch.float32 or torch.bfloat16; gate_act: a name of ACTIVATIONS; an eps of 0: no norm in that place."""
    import torch
    code = {torch.float32: PQL_F32, torch.bfloat16: PQL_BF16}.get(dtype)
    if code is None:
        raise TypeError("rows are float32 or bfloat16, not %s" % dtype)
    return PqlResidualShape(batch, steps, dim, groups, code, gate_cols, ACTIVATIONS[gate_act], eps_post, eps_pre, scale_x, scale_y)


class _Residual:
    def __init__(self, struct, shape, x, y, gate, post, pre, what):
        n, dim, dtype = shape.batch * shape.steps, shape.dim, shape.dtype
        self.key = (n, dim, dtype)
        self.tensors = (x, y, gate, post, pre)
        self.dev = _one_device(what, *self.tensors)
        self.c = struct()
        self.c.x = _rows(x, self.key, what + ": x")
        self.c.y = _rows(y, self.key, what + ": y")
        self.c.gate = _rows(gate, (n, shape.gate_cols, dtype), what + ": gate")
        self.c.post, self.c.pre = _floats(post, dim, what + ": post"), _floats(pre, dim, what + ": pre")
        self.shape = bytes(shape)
        self.ref = C.byref(self.c)


class ResidualInput(_Residual):
    """What pql_residual_forward reads: x, y [batch, steps, dim], gate [batch, steps, gate_cols], post, pre: float32 [dim],
    lengths: int32 [batch]; each may be None."""

    def __init__(self, shape, x=None, y=None, gate=None, post=None, pre=None, lengths=None):
        super().__init__(PqlResidualInput, shape, x, y, gate, post, pre, "ResidualInput")
        self.lengths = lengths
        self.c.lengths = _ints(lengths, shape.batch, "ResidualInput: lengths")
        _one_device("ResidualInput", x, y, lengths)


class ResidualGrad(_Residual):
    """Where the gradients go; the shapes of the inputs, each may be None."""

    def __init__(self, shape, x=None, y=None, gate=None, post=None, pre=None):
        super().__init__(PqlResidualGrad, shape, x, y, gate, post, pre, "ResidualGrad")


def ffn_shape(x, gate, act: str) -> PqlFfnShape:
    """The shape of a call from its tokens [batch, steps, dim] and its gate's weights [hidden, dim]; act: of ACTIVATIONS."""
    if x.dim() != 3 or gate.dim() != 2 or gate.shape[1] != x.shape[2] or gate.dtype != x.dtype:
        raise ValueError("x: [batch, steps, dim], gate: [hidden, dim], of one type")
    return PqlFfnShape(*x.shape, gate.shape[0], S.dtype_code(x), ACTIVATIONS[act])


class _Ffn:
    def __init__(self, struct, shape, x, gate, up, down, what):
        n, dim, hidden, dtype = shape.batch * shape.steps, shape.dim, shape.hidden, shape.dtype
        self.key = (n, dim, dtype)
        self.tensors = (x, gate, up, down)
        self.dev = _one_device(what, *self.tensors)
        self.c = struct()
        self.c.x = _rows(x, self.key, what + ": x")
        self.c.gate = _rows(gate, (hidden, dim, dtype), what + ": gate")
        self.c.up = _rows(up, (hidden, dim, dtype), what + ": up")
        self.c.down = _rows(down, (dim, hidden, dtype), what + ": down")
        self.shape = bytes(shape)
        self.ref = C.byref(self.c)


class FfnInput(_Ffn):
    """What pql_ffn_forward reads: x [batch, steps, dim], gate and up [hidden, dim], down [dim, hidden], lengths int32 [batch]
    or None."""

    def __init__(self, shape, x, gate, up, down, lengths=None):
        super().__init__(PqlFfnInput, shape, x, gate, up, down, "FfnInput")
        self.lengths, self.sizes = lengths, {}
        self.c.lengths = _ints(lengths, shape.batch, "FfnInput: lengths")
        _one_device("FfnInput", x, lengths)


class FfnGrad(_Ffn):
    """Where the gradients go; the shapes of the inputs, each may be None."""

    def __init__(self, shape, x=None, gate=None, up=None, down=None):
        super().__init__(PqlFfnGrad, shape, x, gate, up, down, "FfnGrad")


class BlockContext(S.StudentContext):
    """A context whose methods are the entry points of a block beside those of ``StudentContext``."""

    def __init__(self, cfg: B.PqlConfig = None):
        load_library()
        super().__init__(cfg)

    # ---- host queries
    def embed_workspace_bytes(self, shape: PqlEmbedShape) -> int:
        return self.lib.pql_embed_workspace_bytes(C.byref(shape))

    def residual_workspace_bytes(self, shape: PqlResidualShape) -> int:
        return self.lib.pql_residual_workspace_bytes(C.byref(shape))

    def ffn_saved_bytes(self, shape: PqlFfnShape) -> int:
        return self.lib.pql_ffn_saved_bytes(C.byref(shape))

    def ffn_workspace_bytes(self, shape: PqlFfnShape, call: int) -> int:
        return self.lib.pql_ffn_workspace_bytes(C.byref(shape), call)

    # ---- device calls
    @staticmethod
    def _embed(s, tokens, lengths, table, out):
        n = s.batch * s.steps
        return (C.byref(s), _ints(tokens, n * s.per_row, "tokens"), _ints(lengths, s.batch, "lengths"),
                _ref(table, (s.vocab, s.dim, s.dtype), "table"), _ref(out, (n, s.dim, s.dtype), "rows"))

    def pql_embed_forward(self, shape, tokens, lengths, table: Rows, out: Rows, stream=None):
        given = self._embed(shape, tokens, lengths, table, out)
        stream = _stream(stream, tokens.get_device(), table.dev, out.dev, *_dev(lengths))
        self._check(self.lib.pql_embed_forward(self.h, *given, stream))

    def pql_embed_backward(self, shape, tokens, lengths, out_grad: Rows, table_grad: Rows, workspace, stream=None):
        s, t, n, table, rows = self._embed(shape, tokens, lengths, table_grad, out_grad)
        space = _space(workspace, self.lib.pql_embed_workspace_bytes(s), "workspace")
        stream = _stream(stream, tokens.get_device(), out_grad.dev, table_grad.dev, *_dev(lengths, workspace))
        self._check(self.lib.pql_embed_backward(self.h, s, t, n, rows, table, space, stream))

    @staticmethod
    def _of(shape, *described):
        for d in described:
            if d.shape != bytes(shape):
                raise ValueError("tensors and shape of the call do not agree")

    def pql_residual_forward(self, shape, given: ResidualInput, sum: Rows, next: Rows, stream=None):
        self._of(shape, given)
        total, after = _ref(sum, given.key, "sum"), _ref(next, given.key, "next")
        stream = _stream(stream, given.dev, *(r.dev for r in (sum, next) if r is not None))
        self._check(self.lib.pql_residual_forward(self.h, C.byref(shape), given.ref, total, after, stream))

    def pql_residual_backward(self, shape, given: ResidualInput, sum_grad: Rows, next_grad: Rows, grads: ResidualGrad, workspace,
                              stream=None):
        self._of(shape, given, grads)
        total, after = _ref(sum_grad, given.key, "sum_grad"), _ref(next_grad, given.key, "next_grad")
        used = workspace is not None and (grads.c.post or grads.c.pre)
        space = _space(workspace, self.residual_workspace_bytes(shape) if used else 0, "workspace")
        stream = _stream(stream, given.dev, grads.dev, *(r.dev for r in (sum_grad, next_grad) if r is not None), *_dev(workspace))
        self._check(self.lib.pql_residual_backward(self.h, C.byref(shape), given.ref, total, after, grads.ref, space, stream))

    def _spaces(self, shape, given, saved, workspace, call):
        need = given.sizes.get(call)                # asked for once for each description
        if need is None:
            rows = shape.batch * shape.steps        # none: nothing of either is used
            need = given.sizes[call] = (self.ffn_saved_bytes(shape), self.ffn_workspace_bytes(shape, call)) if rows else (0, 0)
        return _space(saved, need[0], "saved"), _space(workspace, need[1], "workspace")

    def pql_ffn_forward(self, shape, given: FfnInput, out: Rows, saved, workspace, stream=None):
        self._of(shape, given)
        rows = _ref(out, given.key, "out")
        kept, space = self._spaces(shape, given, saved, workspace, FFN_FORWARD)
        stream = _stream(stream, given.dev, *(() if out is None else (out.dev,)), *_dev(saved, workspace))
        self._check(self.lib.pql_ffn_forward(self.h, C.byref(shape), given.ref, rows, kept, space, stream))

    def pql_ffn_backward(self, shape, given: FfnInput, saved, out_grad: Rows, grads: FfnGrad, workspace, stream=None):
        self._of(shape, given, grads)
        rows = _ref(out_grad, given.key, "out_grad")
        kept, space = self._spaces(shape, given, saved, workspace, FFN_BACKWARD_ALONE if saved is None else FFN_BACKWARD)
        stream = _stream(stream, given.dev, grads.dev, *(() if out_grad is None else (out_grad.dev,)), *_dev(saved, workspace))
        self._check(self.lib.pql_ffn_backward(self.h, C.byref(shape), given.ref, kept, rows, grads.ref, space, stream))
