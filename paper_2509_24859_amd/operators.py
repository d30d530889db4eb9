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
ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1
SCALING_NONE, SCALING_LINEAR, SCALING_NTK, SCALING_BY_PARTS = range(4)
NORM_MAX_COLS = 8192
ATTENTION_MAX_HEAD = 128
_ACTS = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH, "silu": ACT_SILU}
_NORMS = {"none": NORM_NONE, "rms": NORM_RMS, "layer": NORM_LAYER}
_LAYOUTS = {"half": ROTARY_HALF, "interleaved": ROTARY_INTERLEAVED}
_SCALINGS = {"none": SCALING_NONE, "linear": SCALING_LINEAR, "ntk": SCALING_NTK, "by_parts": SCALING_BY_PARTS}
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


def _heads(ctx, t, shape, dtype, name):
    """(address, distance of tokens, distance of heads) of [tokens][heads][head] whose channels are contiguous; for None (None, 0, 0)."""
    if t is None:
        return None, 0, 0
    if t.get_device() != ctx.index:
        raise _elsewhere(ctx, t, name)
    if t.dtype is not dtype or t.shape != shape:
        raise HarpError(ERR_SHAPE, "%s: %s of %s is wanted, got %s of %s" % (name, tuple(shape), dtype, tuple(t.shape), t.dtype))
    token, step, channel = t.stride()
    if channel != 1 and shape[2] > 1:
        raise HarpError(ERR_SHAPE, "%s: channels must be contiguous, its strides are %s" % (name, (token, step, channel)))
    return t.data_ptr(), token, step


def _three(t, name):
    if t.dim() != 3:
        raise HarpError(ERR_SHAPE, "%s must be [tokens][heads][head]" % name)


class harp_rotary_args(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("heads", C.c_int32), ("head", C.c_int32), ("turned", C.c_int32), ("type", C.c_int32),
                ("layout", C.c_int32), ("inverse", C.c_int32), ("magnitude", C.c_float), ("X", C.c_void_p), ("x_token", C.c_int64),
                ("x_step", C.c_int64), ("Y", C.c_void_p), ("y_token", C.c_int64), ("y_step", C.c_int64), ("frequency", C.c_void_p),
                ("positions", C.c_void_p), ("first", C.c_int64), ("period", C.c_int64)]


def rotary_frequencies(ctx: Context, turned: int, base=10000.0, scaling="none", factor=1.0, original=0.0, low=1.0, high=32.0):
    """(float64 [turned / 2] on the GPU, magnitude) for harp_rotary; see harp_rotary_frequencies in include/harp.h."""
    out, magnitude = (C.c_double * max(turned // 2, 1))(), C.c_float()
    rc = ctx.lib.harp_rotary_frequencies(turned, base, _named(scaling, _SCALINGS), factor, original, low, high, out, C.byref(magnitude))
    if rc:
        raise HarpError(rc, "frequencies of %s channels: base %s, scaling %s by %s, original %s, low %s, high %s"
                        % (turned, base, scaling, factor, original, low, high))
    return _torch().tensor(list(out), dtype=_torch().float64).to(ctx.device), magnitude.value


def harp_rotary(ctx: Context, x, y, frequencies, positions=None, first=0, period=0, layout="half", magnitude=1.0, inverse=False, stream=None):
    """y = x [tokens][heads][head] with its first 2 * len(frequencies) channels turned; see include/harp.h.  y may be x.
    positions: int64 [tokens], or None: first + t, or first + t % period."""
    _three(x, "x")
    shape, torch = x.shape, _torch()
    turned = 2 * frequencies.numel()
    a = harp_rotary_args(shape[0], shape[1], shape[2], turned, _type(x), _named(layout, _LAYOUTS), int(bool(inverse)), magnitude,
                         *_heads(ctx, x, shape, x.dtype, "x"), *_heads(ctx, y, shape, x.dtype, "y"),
                         _vector(ctx, frequencies, turned // 2, torch.float64, "frequencies"),
                         _vector(ctx, positions, shape[0], torch.int64, "positions"), first, period)
    ctx.check(ctx.lib.harp_rotary(ctx.handle, C.byref(a), _stream(ctx, stream, (x, y, frequencies, positions))))


class harp_attention(C.Structure):
    _fields_ = [("tokens_q", C.c_int64), ("tokens_k", C.c_int64), ("batch", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head", C.c_int32), ("type", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float), ("q_begin", C.c_void_p),
                ("k_begin", C.c_void_p), ("k_count", C.c_void_p), ("Q", C.c_void_p), ("K", C.c_void_p), ("V", C.c_void_p),
                ("q_token", C.c_int64), ("q_step", C.c_int64), ("k_token", C.c_int64), ("k_step", C.c_int64), ("v_token", C.c_int64),
                ("v_step", C.c_int64), ("O", C.c_void_p), ("o_token", C.c_int64), ("o_step", C.c_int64), ("lse", C.c_void_p)]


class harp_attention_grads(C.Structure):
    _fields_ = [("dO", C.c_void_p), ("do_token", C.c_int64), ("do_step", C.c_int64), ("dQ", C.c_void_p), ("dK", C.c_void_p),
                ("dV", C.c_void_p), ("dq_token", C.c_int64), ("dq_step", C.c_int64), ("dk_token", C.c_int64), ("dk_step", C.c_int64),
                ("dv_token", C.c_int64), ("dv_step", C.c_int64)]


def attention_workspace(ctx: Context, tokens_q: int, tokens_k: int, batch: int, heads: int, kv_heads: int, head: int):
    """What harp_attention_forward and harp_attention_backward need for Q [tokens_q][heads][head] and K [tokens_k][kv_heads][head]."""
    a = harp_attention(tokens_q, tokens_k, batch, heads, kv_heads, head)
    size = ctx.lib.harp_attention_workspace_bytes(ctx.handle, C.byref(a))
    if size == 0:
        raise HarpError(ERR_SHAPE, ctx.lib.harp_last_error(ctx.handle).decode())
    return _torch().empty(size, dtype=_torch().uint8, device=ctx.device)


def _attention(ctx, q, k, v, o, lse, q_begin, k_begin, k_count, batch, causal, scale):
    for t, name in ((q, "q"), (k, "k")):
        _three(t, name)
    torch, t = _torch(), q.dtype
    (tq, heads, head), (tk, kv_heads, _) = q.shape, k.shape
    for begin, name in ((q_begin, "q_begin"), (k_begin, "k_begin")):
        if begin is not None:
            if batch is not None and batch != begin.numel() - 1:
                raise HarpError(ERR_SHAPE, "%s has %d entries for %d sequences" % (name, begin.numel(), batch))
            batch = begin.numel() - 1
    batch = 1 if batch is None else batch
    i32, of_k = torch.int32, (tk, kv_heads, head)
    qp, kp, vp, op = (_heads(ctx, x, s, t, n) for x, s, n in ((q, q.shape, "q"), (k, of_k, "k"), (v, of_k, "v"), (o, q.shape, "o")))
    return harp_attention(tq, tk, batch, heads, kv_heads, head, _type(q, (BF16, F16)), int(bool(causal)),
                          head ** -0.5 if scale is None else scale, _vector(ctx, q_begin, batch + 1, i32, "q_begin"),
                          _vector(ctx, k_begin, batch + 1, i32, "k_begin"), _vector(ctx, k_count, batch, i32, "k_count"),
                          qp[0], kp[0], vp[0], *qp[1:], *kp[1:], *vp[1:], *op, _vector(ctx, lse, heads * tq, torch.float32, "lse"))


def harp_attention_forward(ctx: Context, q, k, v, o, lse=None, q_begin=None, k_begin=None, k_count=None, batch=None, causal=False, scale=None,
                           workspace=None, stream=None):
    """o = softmax(scale q k^T) v per sequence and head; see include/harp.h.  q, o: [tokens][heads][head], k, v:
    [tokens][kv heads][head]; begins: int32 [sequences + 1] on the GPU, or None: `batch` (1) sequences of equal length; k_count:
    int32 [sequences], the keys that each uses; lse: float32 [heads][tokens], or None; scale: head^-0.5 if None."""
    a = _attention(ctx, q, k, v, o, lse, q_begin, k_begin, k_count, batch, causal, scale)
    tensors = (q, k, v, o, lse, q_begin, k_begin, k_count, workspace)
    ctx.check(ctx.lib.harp_attention_forward(ctx.handle, C.byref(a), *_workspace(ctx, workspace), _stream(ctx, stream, tensors)))


def harp_attention_backward(ctx: Context, q, k, v, o, lse, do, dq, dk, dv, q_begin=None, k_begin=None, k_count=None, batch=None, causal=False,
                            scale=None, workspace=None, stream=None):
    """The gradients of harp_attention_forward, given do and what that call wrote; dq, dk, dv may be None; see include/harp.h."""
    a = _attention(ctx, q, k, v, o, lse, q_begin, k_begin, k_count, batch, causal, scale)
    t = q.dtype
    d = [_heads(ctx, x, s, t, n) for x, s, n in ((do, q.shape, "do"), (dq, q.shape, "dq"), (dk, k.shape, "dk"), (dv, k.shape, "dv"))]
    g = harp_attention_grads(*d[0], d[1][0], d[2][0], d[3][0], *d[1][1:], *d[2][1:], *d[3][1:])
    tensors = (q, k, v, o, lse, do, dq, dk, dv, q_begin, k_begin, k_count, workspace)
    ctx.check(ctx.lib.harp_attention_backward(ctx.handle, C.byref(a), C.byref(g), *_workspace(ctx, workspace), _stream(ctx, stream, tensors)))


class harp_gated(C.Structure):
    _fields_ = [("M", C.c_int64), ("F", C.c_int64), ("K", C.c_int64), ("type", C.c_int32), ("act", C.c_int32), ("X", C.c_void_p),
                ("ldx", C.c_int64), ("W", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p), ("H", C.c_void_p), ("ldh", C.c_int64),
                ("Z", C.c_void_p), ("ldz", C.c_int64)]


class harp_gated_grads(C.Structure):
    _fields_ = [("M", C.c_int64), ("F", C.c_int64), ("N", C.c_int64), ("type", C.c_int32), ("act", C.c_int32), ("dY", C.c_void_p),
                ("lddy", C.c_int64), ("W", C.c_void_p), ("ldw", C.c_int64), ("Z", C.c_void_p), ("ldz", C.c_int64), ("dZ", C.c_void_p),
                ("lddz", C.c_int64), ("H", C.c_void_p), ("ldh", C.c_int64)]


def gated_workspace(ctx: Context, tokens: int, width: int, channels: int):
    """What harp_gated_forward (x [tokens][channels], w [2 width][channels]) and harp_gated_grad (dy [tokens][channels],
    w [channels][width]) need."""
    size = ctx.lib.harp_gated_workspace_bytes(ctx.handle, tokens, width, channels)
    if size == 0:
        raise HarpError(ERR_SHAPE, "sizes out of range: %s tokens, width %s, %s channels" % (tokens, width, channels))
    return _torch().empty(size, dtype=_torch().uint8, device=ctx.device)


def harp_gated_forward(ctx: Context, x, w, h, bias=None, act="silu", z=None, workspace=None, stream=None):
    """Z = x w^T + bias,  h = act(Z's first half) * Z's second half; see include/harp.h.  w: [2 width][channels], the gate's rows
    first; z: receives Z, or None."""
    _two(x, w, "x", "w")
    (m, k), t = x.shape, x.dtype
    if w.shape[0] % 2:
        raise HarpError(ERR_SHAPE, "w has an odd number of rows, %d" % w.shape[0])
    f = w.shape[0] // 2
    tensors = (x, w, h, bias, z, workspace)
    a = harp_gated(m, f, k, _type(x, (BF16, F16)), _named(act, _ACTS), *_matrix(ctx, x, (m, k), t, "x"), *_matrix(ctx, w, (2 * f, k), t, "w"),
                   _vector(ctx, bias, 2 * f, t, "bias"), *_matrix(ctx, h, (m, f), t, "h"), *_matrix(ctx, z, (m, 2 * f), t, "z"))
    ctx.check(ctx.lib.harp_gated_forward(ctx.handle, C.byref(a), *_workspace(ctx, workspace), _stream(ctx, stream, tensors)))


def harp_gated_grad(ctx: Context, dy, w, z, dz, act="silu", h=None, workspace=None, stream=None):
    """dH = dy w (w [outputs][width], or None: dy is dH),  dz = dH back through the gate,  h = act(gate) * up again; see include/harp.h."""
    _two(dy, z, "dy", "z")
    (m, n), f, t = dy.shape, z.shape[1] // 2, dy.dtype
    n = f if w is None else n
    tensors = (dy, w, z, dz, h, workspace)
    a = harp_gated_grads(m, f, n, _type(dy, (BF16, F16)), _named(act, _ACTS), *_matrix(ctx, dy, (m, n), t, "dy"),
                         *_matrix(ctx, w, (n, f), t, "w"), *_matrix(ctx, z, (m, 2 * f), t, "z"), *_matrix(ctx, dz, (m, 2 * f), t, "dz"),
                         *_matrix(ctx, h, (m, f), t, "h"))
    ctx.check(ctx.lib.harp_gated_grad(ctx.handle, C.byref(a), *_workspace(ctx, workspace), _stream(ctx, stream, tensors)))
