"""ctypes binding of the operators of a stage's training step in include/harp.h.

Tensors in, tensors out: the functions here check what they are given, fill in the structs of the C ABI
and call it on torch's current stream (or `stream`).  They allocate nothing and compute nothing; outputs
and workspaces are the caller's.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C

from .binding import ERR_INVALID_ARG, ERR_SHAPE, Context, HarpError, _torch

F32, BF16, F16 = 0, 1, 2
STATE_F32, STATE_8BIT = 32, 8
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = range(5)
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GATE_LINEAR, GATE_SIGMOID = 0, 1
NORM_MAX_COLS = 8192
_ACTS = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH, "silu": ACT_SILU}
_NORMS = {"none": NORM_NONE, "rms": NORM_RMS, "layer": NORM_LAYER}
_GATES = {"none": GATE_LINEAR, "linear": GATE_LINEAR, "sigmoid": GATE_SIGMOID}
ADAMW_BLOCK = 256           # elements that share an exponent in an 8-bit state

_types = {}


def _type(t, allowed=(F32, BF16, F16)) -> int:
    """The ABI's number of a tensor's type."""
    if not _types:
        torch = _torch()
        _types.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    code = _types.get(t.dtype, -1)
    if code not in allowed:
        raise HarpError(ERR_INVALID_ARG, "a tensor of %s is not taken here" % t.dtype)
    return code


def _elsewhere(ctx, t, name):
    return HarpError(ERR_INVALID_ARG, "%s is on %s, the context is on %s" % (name, t.device, ctx.device))


def _vector(ctx, t, n, dtype, name):
    """The address of a contiguous vector of n elements, or None."""
    if t is None:
        return None
    if t.get_device() != ctx.index:
        raise _elsewhere(ctx, t, name)
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        raise HarpError(ERR_SHAPE, "%s: %d contiguous elements of %s are wanted, got %s of %s"
                        % (name, n, dtype, tuple(t.shape), t.dtype))
    return t.data_ptr()


def _named(value, names):
    """A constant of the ABI, by its number or by its name."""
    if isinstance(value, str):
        if value not in names:
            raise HarpError(ERR_INVALID_ARG, "%r is none of %s" % (value, ", ".join(names)))
        return names[value]
    return int(value)


def _matrix(ctx, t, shape, dtype, name):
    """(address, leading dimension) of a matrix whose rows are contiguous; (None, columns) for None."""
    if t is None:
        return None, shape[1]
    if t.get_device() != ctx.index:
        raise _elsewhere(ctx, t, name)
    if t.dtype is not dtype or t.shape != shape:
        raise HarpError(ERR_SHAPE, "%s: %s of %s is wanted, got %s of %s" % (name, tuple(shape), dtype, tuple(t.shape), t.dtype))
    cols = shape[1]
    if t.is_contiguous():
        return t.data_ptr(), cols
    rows = shape[0]
    row, col = t.stride()
    if (col != 1 and cols > 1) or (row < cols and rows > 1):
        raise HarpError(ERR_SHAPE, "%s: rows must be contiguous and apart, its strides are %s" % (name, (row, col)))
    return t.data_ptr(), row if row > cols else cols


def _current(ctx: Context) -> int:
    """The handle of torch's current stream."""
    raw = getattr(_torch()._C, "_cuda_getCurrentRawStream", None)      # without an object around it
    return raw(ctx.index) if raw else int(_torch().cuda.current_stream(ctx.device).cuda_stream)


def _stream(ctx: Context, stream, tensors):
    """The stream's handle.  Tensors used on another stream than torch's current one are recorded there, so that
    their memory is not handed out again before the call has run."""
    if stream is None:
        return _current(ctx)
    if stream != _torch().cuda.current_stream(ctx.device):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
    return int(stream.cuda_stream)


def _workspace(ctx, w):
    if w is None:
        return None, 0
    if w.get_device() != ctx.index:
        raise _elsewhere(ctx, w, "the workspace")
    return w.data_ptr(), w.numel() * w.element_size()


class harp_linear(C.Structure):
    _fields_ = [("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64), ("type", C.c_int32), ("act", C.c_int32),
                ("X", C.c_void_p), ("ldx", C.c_int64), ("W", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p),
                ("residual", C.c_void_p), ("ldr", C.c_int64), ("Y", C.c_void_p), ("ldy", C.c_int64),
                ("Z", C.c_void_p), ("ldz", C.c_int64)]


class harp_linear_input(C.Structure):
    _fields_ = [("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64), ("type", C.c_int32), ("act", C.c_int32),
                ("dY", C.c_void_p), ("lddy", C.c_int64), ("W", C.c_void_p), ("ldw", C.c_int64), ("Z", C.c_void_p),
                ("ldz", C.c_int64), ("residual", C.c_void_p), ("ldr", C.c_int64), ("dX", C.c_void_p), ("lddx", C.c_int64)]


class harp_linear_weight(C.Structure):
    _fields_ = [("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64), ("type", C.c_int32), ("dw_type", C.c_int32),
                ("accumulate", C.c_int32), ("dY", C.c_void_p), ("lddy", C.c_int64), ("X", C.c_void_p), ("ldx", C.c_int64),
                ("dW", C.c_void_p), ("lddw", C.c_int64), ("dbias", C.c_void_p)]


def linear_workspace(ctx: Context, tokens: int, outputs: int, inputs: int):
    """What harp_linear_forward, harp_linear_grad_input and harp_linear_grad_weight need for X [tokens][inputs] and
    W [outputs][inputs]."""
    size = ctx.lib.harp_linear_workspace_bytes(ctx.handle, tokens, outputs, inputs)
    if size == 0:
        raise HarpError(ERR_SHAPE, "sizes out of range: %s tokens, %s outputs, %s inputs" % (tokens, outputs, inputs))
    return _torch().empty(size, dtype=_torch().uint8, device=ctx.device)


def _two(a, b, name_a, name_b):
    if a.dim() != 2 or b.dim() != 2:
        raise HarpError(ERR_SHAPE, "%s and %s must be matrices" % (name_a, name_b))


def harp_linear_forward(ctx: Context, x, w, y, bias=None, act="none", residual=None, z=None, workspace=None, stream=None):
    """Z = x w^T + bias,  y = act(Z) + residual; see include/harp.h.  z: receives Z, or None."""
    _two(x, w, "x", "w")
    (m, k), n, t = x.shape, w.shape[0], x.dtype
    tensors, out = (x, w, y, bias, residual, z, workspace), (m, n)
    a = harp_linear(m, n, k, _type(x, (BF16, F16)), _named(act, _ACTS), *_matrix(ctx, x, (m, k), t, "x"),
                    *_matrix(ctx, w, (n, k), t, "w"), _vector(ctx, bias, n, t, "bias"),
                    *_matrix(ctx, residual, out, t, "residual"), *_matrix(ctx, y, out, t, "y"), *_matrix(ctx, z, out, t, "z"))
    ctx.check(ctx.lib.harp_linear_forward(ctx.handle, C.byref(a), *_workspace(ctx, workspace), _stream(ctx, stream, tensors)))


def harp_linear_grad_input(ctx: Context, dy, w, dx, act="none", z=None, residual=None, workspace=None, stream=None):
    """dx = (dy w) * act'(z) + residual; see include/harp.h."""
    _two(dy, w, "dy", "w")
    (m, n), k, t = dy.shape, w.shape[1], dy.dtype
    tensors, out = (dy, w, dx, z, residual, workspace), (m, k)
    a = harp_linear_input(m, n, k, _type(dy, (BF16, F16)), _named(act, _ACTS), *_matrix(ctx, dy, (m, n), t, "dy"),
                          *_matrix(ctx, w, (n, k), t, "w"), *_matrix(ctx, z, out, t, "z"),
                          *_matrix(ctx, residual, out, t, "residual"), *_matrix(ctx, dx, out, t, "dx"))
    ctx.check(ctx.lib.harp_linear_grad_input(ctx.handle, C.byref(a), *_workspace(ctx, workspace), _stream(ctx, stream, tensors)))


def harp_linear_grad_weight(ctx: Context, dy, x, dw, dbias=None, accumulate=False, workspace=None, stream=None):
    """dw = dy^T x,  dbias = column sums of dy, added to what they hold with `accumulate`; see include/harp.h."""
    _two(dy, x, "dy", "x")
    (m, n), k, t = dy.shape, x.shape[1], dy.dtype
    tensors = (dy, x, dw, dbias, workspace)
    a = harp_linear_weight(m, n, k, _type(dy, (BF16, F16)), _type(dw), int(bool(accumulate)), *_matrix(ctx, dy, (m, n), t, "dy"),
                           *_matrix(ctx, x, (m, k), t, "x"), *_matrix(ctx, dw, (n, k), dw.dtype, "dw"),
                           _vector(ctx, dbias, n, _torch().float32, "dbias"))
    ctx.check(ctx.lib.harp_linear_grad_weight(ctx.handle, C.byref(a), *_workspace(ctx, workspace), _stream(ctx, stream, tensors)))


def harp_act_grad(ctx: Context, dy, z, dz, act, stream=None):
    """dz = dy * act'(z); see include/harp.h."""
    _two(dy, z, "dy", "z")
    (m, n), t = dy.shape, dy.dtype
    tensors, all_of = (dy, z, dz), (m, n)
    ctx.check(ctx.lib.harp_act_grad(ctx.handle, m, n, _type(dy), _named(act, _ACTS), *_matrix(ctx, dy, all_of, t, "dy"),
                                    *_matrix(ctx, z, all_of, t, "z"), *_matrix(ctx, dz, all_of, t, "dz"),
                                    _stream(ctx, stream, tensors)))


class harp_adamw_tensor(C.Structure):
    _fields_ = [("n", C.c_int64), ("state", C.c_int32), ("grad_type", C.c_int32), ("copy_type", C.c_int32),
                ("flags", C.c_int32), ("p", C.c_void_p), ("grad", C.c_void_p), ("copy", C.c_void_p),
                ("m", C.c_void_p), ("v", C.c_void_p), ("m_exp", C.c_void_p), ("v_exp", C.c_void_p),
                ("m_seen", C.c_void_p), ("v_seen", C.c_void_p), ("weight_decay", C.c_double)]


class harp_adamw_hyper(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("step", C.c_int64), ("seed", C.c_uint64), ("grad_scale", C.c_void_p), ("skip", C.c_void_p)]


_ADAMW_NEEDED = frozenset(("p", "grad", "m", "v"))
_ADAMW_KNOWN = _ADAMW_NEEDED | {"copy", "m_exp", "v_exp", "m_seen", "v_seen", "weight_decay"}


class AdamW:
    """harp_adamw_plan / harp_adamw_step / harp_adamw_read_state / harp_adamw_release.

    tensors: one dict per tensor, of contiguous tensors of equal size:
      p             master weights, float32, updated
      grad          float32, bfloat16 or float16
      m, v          moments: both float32, or both uint8 with m_exp, v_exp (uint8, one per 256 elements)
      copy          optional, bfloat16 or float16: receives the new weights rounded
      m_seen, v_seen  optional, bfloat16: where read_state() puts the values of 8-bit moments
      weight_decay  optional, 0 if absent
    The tensors must stay where they are; this object holds on to them."""

    def __init__(self, ctx: Context, tensors, stream=None):
        torch = _torch()
        f32, u8, bf16 = torch.float32, torch.uint8, torch.bfloat16
        self.ctx, self.handle = ctx, None
        self.tensors = [dict(t) for t in tensors]
        array = (harp_adamw_tensor * max(len(self.tensors), 1))()
        for a, t in zip(array, self.tensors):
            if not (_ADAMW_NEEDED <= t.keys() <= _ADAMW_KNOWN):
                raise HarpError(ERR_INVALID_ARG, "a tensor's entry needs p, grad, m and v, and knows no %s"
                                % (", ".join(sorted(t.keys() - _ADAMW_KNOWN)) or "other"))
            get = t.get
            p, grad, m, copy = t["p"], t["grad"], t["m"], get("copy")
            n = a.n = p.numel()
            eight = m.dtype is u8
            kind, a.state = (u8, STATE_8BIT) if eight else (f32, STATE_F32)
            a.p = _vector(ctx, p, n, f32, "p")
            a.grad_type = _type(grad)
            a.grad = _vector(ctx, grad, n, grad.dtype, "grad")
            a.m, a.v = _vector(ctx, m, n, kind, "m"), _vector(ctx, t["v"], n, kind, "v")
            if eight:
                blocks = -(-n // ADAMW_BLOCK)
                if get("m_exp") is None or get("v_exp") is None:
                    raise HarpError(ERR_INVALID_ARG, "8-bit moments need m_exp and v_exp")
                a.m_exp = _vector(ctx, t["m_exp"], blocks, u8, "m_exp")
                a.v_exp = _vector(ctx, t["v_exp"], blocks, u8, "v_exp")
            if copy is not None:
                a.copy_type = _type(copy, (BF16, F16))
                a.copy = _vector(ctx, copy, n, copy.dtype, "copy")
            a.m_seen = _vector(ctx, get("m_seen"), n, bf16, "m_seen")
            a.v_seen = _vector(ctx, get("v_seen"), n, bf16, "v_seen")
            a.weight_decay = get("weight_decay", 0.0)
        nbytes = ctx.lib.harp_adamw_plan_bytes(array, len(self.tensors))
        self.buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=ctx.device)
        self.home = _current(ctx)           # the stream that buf is handed out again on
        h = C.c_void_p()
        ctx.check(ctx.lib.harp_adamw_plan(ctx.handle, array, len(self.tensors), self.buf.data_ptr(),
                                          self.buf.numel(), C.byref(h), _stream(ctx, stream, [self.buf])))
        self.handle = h

    def step(self, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=None, skip=None, seed=0, stream=None):
        """One step.  grad_scale: a float32 scalar on the GPU that gradients are multiplied by; skip: an int32 one,
        not 0 leaves everything as it is; seed: of the rounding to 8 bits, another one every step.  In a captured graph
        lr, step and seed are those of the capture at every replay."""
        torch = _torch()
        hyper = harp_adamw_hyper(lr, beta1, beta2, eps, step, seed & ((1 << 64) - 1),
                                 _vector(self.ctx, grad_scale, 1, torch.float32, "grad_scale"),
                                 _vector(self.ctx, skip, 1, torch.int32, "skip"))
        self.ctx.check(self.ctx.lib.harp_adamw_step(self.ctx.handle, self.handle, C.byref(hyper),
                                                    self._on_stream(stream, grad_scale, skip)))

    def read_state(self, stream=None):
        """The values that the 8-bit moments stand for, into m_seen and v_seen."""
        self.ctx.check(self.ctx.lib.harp_adamw_read_state(self.ctx.handle, self.handle, self._on_stream(stream)))

    def _on_stream(self, stream, *more):
        """The stream's handle.  On another stream than the current one, or than the one that the plan's memory comes from,
        that memory and the tensors are recorded there: the object may be dropped before the call has run."""
        current = _current(self.ctx)
        handle = current if stream is None else int(stream.cuda_stream)
        if handle != current or handle != self.home:
            if stream is None:
                stream = _torch().cuda.current_stream(self.ctx.device)
            held = [x for t in self.tensors for x in t.values() if hasattr(x, "record_stream")]
            for t in (self.buf, *held, *more):
                if t is not None:
                    t.record_stream(stream)
        return handle

    def release(self):
        if self.handle:
            self.ctx.lib.harp_adamw_release(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.release()
        except Exception:
            pass


class harp_norm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int32), ("type", C.c_int32), ("after", C.c_int32), ("before", C.c_int32),
                ("eps_after", C.c_float), ("eps_before", C.c_float), ("w_after", C.c_void_p), ("b_after", C.c_void_p),
                ("w_before", C.c_void_p), ("b_before", C.c_void_p), ("scale", C.c_void_p), ("gate", C.c_void_p),
                ("ldgate", C.c_int64), ("rows_per_gate", C.c_int64), ("gate_act", C.c_int32)]


class harp_norm_grads(C.Structure):
    _fields_ = [("dh", C.c_void_p), ("dz", C.c_void_p), ("h", C.c_void_p), ("y", C.c_void_p), ("lddh", C.c_int64),
                ("lddz", C.c_int64), ("ldh", C.c_int64), ("ldy", C.c_int64), ("dx", C.c_void_p), ("dy", C.c_void_p),
                ("dgate", C.c_void_p), ("lddx", C.c_int64), ("lddy", C.c_int64), ("lddgate", C.c_int64),
                ("dw_after", C.c_void_p), ("db_after", C.c_void_p), ("dw_before", C.c_void_p), ("db_before", C.c_void_p),
                ("dscale", C.c_void_p), ("accumulate", C.c_int32)]


def _norm(ctx, rows, cols, dtype, after, before, eps, gate, rows_per_gate, gate_act, scale, w_after, b_after, w_before, b_before):
    f32 = _torch().float32
    n = harp_norm(rows, cols, _types[dtype], _named(after, _NORMS), _named(before, _NORMS), eps, eps,
                  _vector(ctx, w_after, cols, f32, "w_after"), _vector(ctx, b_after, cols, f32, "b_after"),
                  _vector(ctx, w_before, cols, f32, "w_before"), _vector(ctx, b_before, cols, f32, "b_before"),
                  _vector(ctx, scale, cols, f32, "scale"))
    n.gate_act = _named(gate_act, _GATES)
    if gate is not None:
        if rows_per_gate < 1:
            raise HarpError(ERR_SHAPE, "rows_per_gate must be at least 1")
        n.gate, n.ldgate = _matrix(ctx, gate, (-(-rows // rows_per_gate), cols), dtype, "gate")
        n.rows_per_gate = rows_per_gate
    return n


def harp_norm_forward(ctx: Context, x, y, h, z, after="rms", before="rms", gate=None, rows_per_gate=1, gate_act="linear",
                      scale=None, w_after=None, b_after=None, w_before=None, b_before=None, eps=1e-5, stream=None):
    """h = x + scale * gate * after(y),  z = before(h); see include/harp.h.  x, y, h, z: [rows][cols] or None."""
    first = x if x is not None else y
    if first is None or first.dim() != 2:
        raise HarpError(ERR_INVALID_ARG, "x or y is wanted, as a matrix")
    _type(first)
    all_of, dtype = first.shape, first.dtype
    rows, cols = all_of
    tensors = (x, y, h, z, gate, scale, w_after, b_after, w_before, b_before)
    n = _norm(ctx, rows, cols, dtype, after, before, eps, gate, rows_per_gate, gate_act, scale, w_after, b_after, w_before, b_before)
    ctx.check(ctx.lib.harp_norm_forward(ctx.handle, C.byref(n), *_matrix(ctx, x, all_of, dtype, "x"), *_matrix(ctx, y, all_of, dtype, "y"),
                                        *_matrix(ctx, h, all_of, dtype, "h"), *_matrix(ctx, z, all_of, dtype, "z"),
                                        _stream(ctx, stream, tensors)))


def norm_workspace(ctx: Context, rows: int, cols: int, rows_per_gate: int = 0):
    """What harp_norm_backward needs for these sizes; rows_per_gate 0: no gate."""
    n = harp_norm(rows, cols, F32)
    if rows_per_gate:
        n.gate, n.ldgate, n.rows_per_gate = 256, cols, rows_per_gate     # of its place only that there is one counts
    size = ctx.lib.harp_norm_workspace_bytes(ctx.handle, C.byref(n))
    if size == 0:
        raise HarpError(ERR_SHAPE, ctx.lib.harp_last_error(ctx.handle).decode())
    return _torch().empty(size, dtype=_torch().uint8, device=ctx.device)


def harp_norm_backward(ctx: Context, dh, dz, h, y, dx, dy, after="rms", before="rms", gate=None, rows_per_gate=1, gate_act="linear",
                       scale=None, w_after=None, b_after=None, w_before=None, b_before=None, eps=1e-5, dgate=None, dscale=None,
                       dw_after=None, db_after=None, dw_before=None, db_before=None, accumulate=False, workspace=None, stream=None):
    """The gradients of harp_norm_forward; see include/harp.h.  Whatever is None is not there or not wanted."""
    first = dh if dh is not None else dz
    if first is None or first.dim() != 2:
        raise HarpError(ERR_INVALID_ARG, "dh or dz is wanted, as a matrix")
    _type(first)
    all_of, dtype, f32 = first.shape, first.dtype, _torch().float32
    rows, cols = all_of
    sums = dict(dw_after=dw_after, db_after=db_after, dw_before=dw_before, db_before=db_before, dscale=dscale)
    tensors = (dh, dz, h, y, dx, dy, gate, scale, w_after, b_after, w_before, b_before, dgate, workspace, *sums.values())
    n = _norm(ctx, rows, cols, dtype, after, before, eps, gate, rows_per_gate, gate_act, scale, w_after, b_after, w_before, b_before)
    if dgate is not None and gate is None:
        raise HarpError(ERR_INVALID_ARG, "dgate without a gate")
    g = harp_norm_grads()
    for name, t in (("dh", dh), ("dz", dz), ("h", h), ("y", y), ("dx", dx), ("dy", dy)):
        p, ld = _matrix(ctx, t, all_of, dtype, name)
        setattr(g, name, p)
        setattr(g, "ld" + name, ld)
    g.dgate, g.lddgate = _matrix(ctx, dgate, (-(-rows // rows_per_gate) if dgate is not None else 0, cols), dtype, "dgate")
    for name, t in sums.items():
        setattr(g, name, _vector(ctx, t, cols, f32, name))
    g.accumulate = int(bool(accumulate))
    ctx.check(ctx.lib.harp_norm_backward(ctx.handle, C.byref(n), C.byref(g), *_workspace(ctx, workspace), _stream(ctx, stream, tensors)))
