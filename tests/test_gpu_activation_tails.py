"""Activations and their slopes far below zero, where they are small beside their terms, and at arguments whose square no
float holds.

Tolerances are relative to the result.  What 32 bits cost: the argument of the error function, the exponential or the
logistic function is off by at most four roundings of 2^-24 of itself, and a relative change of the argument z changes the
result by z f'(z) / f(z) times as much, at most 155 at z = -8 (the tanh form's z^3); the functions themselves are within 16
units of the last place: under 1,024 roundings of 2^-24 in all.  A stored result adds half a unit of its last place,
2^-8 or 2^-11 of it (8 and 11 bits of significand), in float16 below 2^-14 2^-25.
"""
import math

import numpy as np
import pytest

ROOM = 1024 * 2.0 ** -24
HALF = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}


def _exact(z, act):
    """Activation and slope in 64 bits, without a difference of nearly equal numbers (z <= -2)."""
    if act == "gelu":
        cdf = 0.5 * math.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * math.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        s = 1 / (1 + math.exp(-c * (z + 0.044715 * z ** 3)))
        return z * s, s + z * s * (1 - s) * c * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + math.exp(-z))
    return z * s, s + z * s * (1 - s)


def _arguments(torch, kind):
    """64 x 64 values of the type in -8 .. -2, in 64 bits."""
    z = np.linspace(-8.0, -2.0, 4096).reshape(64, 64)
    return torch.from_numpy(z).to(kind).double().numpy()


def _close(got, want, kind, what):
    got = got.double().cpu().numpy()
    room = np.abs(want) * (ROOM + HALF[kind]) * (1 + ROOM) + (2.0 ** -25 if kind == "float16" else 0)
    off = np.abs(got - want)
    worst = np.unravel_index(np.argmax(off / room), off.shape)
    assert (off <= room).all(), (what, got[worst], want[worst])


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("copies", [1, 5], ids=["few_tokens", "tiles"])
def test_tails_in_a_product(harp, act, kind, copies):
    """Weights of one: Z is X, and the gradient before the slope is one."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    t = getattr(torch, kind)
    z = np.concatenate([_arguments(torch, t)] * copies)
    x = torch.from_numpy(z).to(t).cuda()
    eye, ones = torch.eye(64, device="cuda").to(t), torch.ones(x.shape, device="cuda", dtype=t)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    ws = ops.linear_workspace(ctx, x.shape[0], 64, 64)
    ops.harp_linear_forward(ctx, x, eye, y, act=act, workspace=ws)
    ops.harp_linear_grad_input(ctx, ones, eye, dx, act=act, z=x, workspace=ws)
    want = np.vectorize(lambda v: _exact(v, act), otypes=[float, float])(z)
    _close(y, want[0], kind, "activation")
    _close(dx, want[1], kind, "slope")
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_tails_of_a_slope_alone(harp, act, kind):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    t = getattr(torch, kind)
    z = _arguments(torch, t)
    x = torch.from_numpy(z).to(t).cuda()
    dz = torch.empty_like(x)
    ops.harp_act_grad(ctx, torch.ones_like(x), x, dz, act)
    _close(dz, np.vectorize(lambda v: _exact(v, act)[1], otypes=[float])(z), kind, "slope")
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_slopes_of_huge_arguments(harp, act, kind):
    """One above and zero below, also where the argument's square or cube is beyond 32 bits; NaN stays NaN (the derivative
    of max(z, 0) is taken to be zero wherever z is not above zero)."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    t = getattr(torch, kind)
    large = [100.0, 1e6, 1e13, 1e18, 5e18, 1e19, 6e19, 1e20, 1e30, 3e38]
    z = torch.tensor([large, [-v for v in large]], dtype=t, device="cuda")
    dz = torch.full_like(z, -7.0)
    ops.harp_act_grad(ctx, torch.ones_like(z), z, dz, act)
    assert (dz[0] == 1).all() and (dz[1] == 0).all(), dz.tolist()
    z.fill_(math.nan)
    ops.harp_act_grad(ctx, torch.ones_like(z), z, dz, act)
    assert (dz == 0).all() if act == "relu" else torch.isnan(dz).all()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("copies", [1, 80], ids=["few_tokens", "tiles"])
def test_huge_arguments_in_a_product(harp, copies):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    z = torch.tensor([[1e20] * 8, [-1e20] * 8, [3e38] * 8, [-3e38] * 8], device="cuda").bfloat16().repeat(copies, 1)
    eye, ones = torch.eye(8, device="cuda").bfloat16(), torch.ones_like(z)
    ws = ops.linear_workspace(ctx, z.shape[0], 8, 8)
    for act in ("relu", "gelu", "gelu_tanh", "silu"):
        y, dx = torch.empty_like(z), torch.empty_like(z)
        ops.harp_linear_forward(ctx, z, eye, y, act=act, workspace=ws)
        ops.harp_linear_grad_input(ctx, ones, eye, dx, act=act, z=z, workspace=ws)
        assert torch.equal(y, z.clamp(min=0)), act
        assert torch.equal(dx, (z > 0).to(dx.dtype)), act
    ctx.close()
