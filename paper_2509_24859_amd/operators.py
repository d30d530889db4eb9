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
ADAMW_BLOCK = 256           # elements that share an exponent in an 8-bit state

_types = {}


def _type(t, allowed=(F32, BF16, F16)) -> int:
    if not _types:
        torch = _torch()
        _types.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    code = _types.get(t.dtype, -1)
    if code not in allowed:
        raise HarpError(ERR_INVALID_ARG, "a tensor of %s is not taken here" % t.dtype)
    return code


def _on(ctx: Context, *tensors):
    for t in tensors:
        if t is not None and t.device != ctx.device:
            raise HarpError(ERR_INVALID_ARG, "a tensor on %s, the context is on %s" % (t.device, ctx.device))


def _vector(t, n, dtype, name):
    """A contiguous vector of n elements, or None."""
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise HarpError(ERR_SHAPE, "%s: %d contiguous elements of %s are wanted, got %s of %s"
                        % (name, n, dtype, tuple(t.shape), t.dtype))
    return t.data_ptr()


def _stream(ctx: Context, stream, tensors):
    """The stream's handle.  Tensors used on another stream than torch's current one are recorded there, so that
    their memory is not handed out again before the call has run."""
    torch = _torch()
    current = torch.cuda.current_stream(ctx.device)
    if stream is None or stream == current:
        return int(current.cuda_stream)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return int(stream.cuda_stream)


class harp_adamw_tensor(C.Structure):
    _fields_ = [("n", C.c_int64), ("state", C.c_int32), ("grad_type", C.c_int32), ("copy_type", C.c_int32),
                ("flags", C.c_int32), ("p", C.c_void_p), ("grad", C.c_void_p), ("copy", C.c_void_p),
                ("m", C.c_void_p), ("v", C.c_void_p), ("m_exp", C.c_void_p), ("v_exp", C.c_void_p),
                ("m_seen", C.c_void_p), ("v_seen", C.c_void_p), ("weight_decay", C.c_double)]


class harp_adamw_hyper(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("step", C.c_int64), ("seed", C.c_uint64), ("grad_scale", C.c_void_p), ("skip", C.c_void_p)]


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
        self.ctx, self.handle = ctx, None
        self.tensors = [dict(t) for t in tensors]
        array = (harp_adamw_tensor * max(len(self.tensors), 1))()
        held = []
        for a, t in zip(array, self.tensors):
            unknown = set(t) - {"p", "grad", "m", "v", "copy", "m_exp", "v_exp", "m_seen", "v_seen", "weight_decay"}
            if unknown or not {"p", "grad", "m", "v"} <= set(t):
                raise HarpError(ERR_INVALID_ARG, "a tensor's entry needs p, grad, m and v, and knows no %s"
                                % (", ".join(sorted(unknown)) or "other"))
            n = t["p"].numel()
            eight = t["m"].dtype == torch.uint8
            kind = torch.uint8 if eight else torch.float32
            a.n, a.state = n, STATE_8BIT if eight else STATE_F32
            a.p = _vector(t["p"], n, torch.float32, "p")
            a.grad_type = _type(t["grad"])
            a.grad = _vector(t["grad"], n, t["grad"].dtype, "grad")
            a.m, a.v = _vector(t["m"], n, kind, "m"), _vector(t["v"], n, kind, "v")
            if eight:
                blocks = -(-n // ADAMW_BLOCK)
                if t.get("m_exp") is None or t.get("v_exp") is None:
                    raise HarpError(ERR_INVALID_ARG, "8-bit moments need m_exp and v_exp")
                a.m_exp = _vector(t["m_exp"], blocks, torch.uint8, "m_exp")
                a.v_exp = _vector(t["v_exp"], blocks, torch.uint8, "v_exp")
            if t.get("copy") is not None:
                a.copy_type = _type(t["copy"], (BF16, F16))
                a.copy = _vector(t["copy"], n, t["copy"].dtype, "copy")
            a.m_seen = _vector(t.get("m_seen"), n, torch.bfloat16, "m_seen")
            a.v_seen = _vector(t.get("v_seen"), n, torch.bfloat16, "v_seen")
            a.weight_decay = float(t.get("weight_decay", 0.0))
            held += [x for x in t.values() if isinstance(x, torch.Tensor)]
        _on(ctx, *held)
        self.held = held
        nbytes = ctx.lib.harp_adamw_plan_bytes(array, len(self.tensors))
        self.buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=ctx.device)
        h = C.c_void_p()
        ctx.check(ctx.lib.harp_adamw_plan(ctx.handle, array, len(self.tensors), self.buf.data_ptr(),
                                          self.buf.numel(), C.byref(h), _stream(ctx, stream, [self.buf])))
        self.handle = h

    def step(self, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=None, skip=None, seed=0, stream=None):
        """One step.  grad_scale: a float32 scalar on the GPU that gradients are multiplied by; skip: an int32 one,
        not 0 leaves everything as it is; seed: of the rounding to 8 bits, another one every step."""
        torch = _torch()
        _on(self.ctx, grad_scale, skip)
        hyper = harp_adamw_hyper(lr, beta1, beta2, eps, step, seed & ((1 << 64) - 1),
                                 _vector(grad_scale, 1, torch.float32, "grad_scale"),
                                 _vector(skip, 1, torch.int32, "skip"))
        self.ctx.check(self.ctx.lib.harp_adamw_step(self.ctx.handle, self.handle, C.byref(hyper),
                                                    self._on_stream(stream, grad_scale, skip)))

    def read_state(self, stream=None):
        """The values that the 8-bit moments stand for, into m_seen and v_seen."""
        self.ctx.check(self.ctx.lib.harp_adamw_read_state(self.ctx.handle, self.handle, self._on_stream(stream)))

    def _on_stream(self, stream, *more):
        if stream is None:
            return _stream(self.ctx, None, ())
        return _stream(self.ctx, stream, [self.buf, *self.held, *more])

    def release(self):
        if self.handle:
            self.ctx.lib.harp_adamw_release(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.release()
        except Exception:
            pass
