"""The AdamW step over many tensors against its formula in 64 bits.

Tolerances: in 32 bits m is two products and a sum, each rounded, with constants rounded to 32 bits: 4 roundings of
2^-24 of (|beta1 m| + |(1 - beta1) g|); v the same with one product more.  The weight is p keep - step m / (root + eps):
2 roundings of |p| and 10 of the quotient.  An 8-bit state's value is one of the two codes around the exact value, so
less than one step away, and the code is the one that the random bits say wherever that is no closer than the 32-bit
value's own error.
"""
import math

import numpy as np
import pytest

EPS24 = 2.0 ** -24
BLOCK = 256
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)


def _decode(code, exponent, top):
    """What 8-bit codes stand for, in 64 bits (numpy)."""
    code = code.astype(np.int64)
    mag = code & 127 if top == 15 else code
    e, f = mag >> 3, mag & 7
    E = np.maximum(np.repeat(exponent.astype(np.int64), BLOCK)[:code.size], 64)
    value = np.where(e > 0, (8 + f) * 2.0 ** (e - 1), f) * 2.0 ** (E - 129 - top)
    value = np.where(E == 255, np.nan, value)
    return np.where(code >> 7, -value, value) if top == 15 else value


def _random_bits(places, seed):
    """16 bits for m and 16 for v per place (splitmix64 of the pair, the half of the place)."""
    with np.errstate(over="ignore"):
        z = (places // 2).astype(np.uint64) * np.uint64(0x9E3779B97F4A7C15) + np.uint64(seed)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    half = (z >> (np.uint64(32) * (places % 2).astype(np.uint64))).astype(np.int64) & 0xFFFFFFFF
    return half & 0xFFFF, half >> 16


def _exact(p, g, m, v, wd, step):
    m = HYPER["beta1"] * m + (1 - HYPER["beta1"]) * g
    v = HYPER["beta2"] * v + (1 - HYPER["beta2"]) * g * g
    u = m / (1 - HYPER["beta1"] ** step) / (np.sqrt(v / (1 - HYPER["beta2"] ** step)) + HYPER["eps"])
    return p * (1 - HYPER["lr"] * wd) - HYPER["lr"] * u, m, v, HYPER["lr"] * u


def _f64(t):
    return t.double().cpu().numpy()


def _tensor(torch, n, state, grad_type, copy_type, seed, lead=0, zero=False):
    """One entry; lead: elements cut off the front of every buffer (alignment)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def cut(t):
        return t[lead:]

    t = {"p": cut(torch.randn(n + lead, generator=gen, device="cuda")),
         "grad": cut((torch.randn(n + lead, generator=gen, device="cuda") * 0.01).to(grad_type))}
    if state == 32:
        t["m"] = cut(torch.randn(n + lead, generator=gen, device="cuda") * (0 if zero else 0.01))
        t["v"] = cut(torch.rand(n + lead, generator=gen, device="cuda") * (0 if zero else 1e-4))
    else:
        blocks = -(-n // BLOCK)
        for name in ("m", "v"):
            t[name] = cut(torch.randint(0, 1 if zero else 256, (n + lead,), generator=gen, device="cuda").to(torch.uint8))
        t["m_exp"] = torch.randint(115, 122, (blocks,), generator=gen, device="cuda").to(torch.uint8) * (not zero)
        t["v_exp"] = torch.randint(106, 114, (blocks,), generator=gen, device="cuda").to(torch.uint8) * (not zero)
        t["m_seen"], t["v_seen"] = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if copy_type is not None:
        t["copy"] = cut(torch.zeros(n + lead, dtype=copy_type, device="cuda"))
    return t


def _codes_fit(code, exponent, exact, top, rnd, slack):
    """Codes and exponents of one tensor against the exact new moment."""
    a = np.abs(exact)
    for b in range(exponent.size):
        x, E = a[b * BLOCK:(b + 1) * BLOCK], int(exponent[b])
        most = max(x.max(), 2.0 ** -63)
        near = [max(64, 127 + math.frexp(most * s / 1.875)[1]) for s in (1 - 1e-6, 1 + 1e-6)]
        near = [e - 1 if most * s <= 1.875 * 2.0 ** (e - 1 - 127) else e for e, s in zip(near, (1 - 1e-6, 1 + 1e-6))]
        assert near[0] <= E <= near[1], (b, E, most, near)
    E = np.repeat(exponent.astype(np.int64), BLOCK)[:code.size]
    least = 2.0 ** (E - 129 - top)
    step = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(a, 1e-300))) - 3), least)
    value = _decode(code, exponent, top)
    assert (np.abs(value - exact) <= step * (1 + 1e-5) + slack).all()
    want = np.floor(a / step + rnd / 65536) * step
    agree = np.abs(np.abs(value) - want) <= 1e-6 * step
    # a wrong code where the fraction is not within the error of the 32-bit value is a fault
    fraction = a / step + rnd / 65536
    close = np.abs(fraction - np.round(fraction)) <= slack / step + 1e-5
    assert (agree | close).all()
    assert close.mean() < 0.01


@pytest.mark.gpu
@pytest.mark.parametrize("state", [32, 8])
@pytest.mark.parametrize("grad", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("lead", [0, 1, 4])
def test_a_step_is_the_formula(harp, state, grad, lead):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    copies = (torch.bfloat16, None, torch.float16)
    sizes = (1, 3, 255, 256, 257, 1000, 4095, 4096, 4097, 20_011, 0, 64)
    tensors = [_tensor(torch, n, state, getattr(torch, grad), copies[i % 3], 100 + i, lead) for i, n in enumerate(sizes)]
    for i, t in enumerate(tensors):
        t["weight_decay"] = 0.1 * (i % 2)
    old = [{k: x.clone() for k, x in t.items() if torch.is_tensor(x)} for t in tensors]
    scale = torch.full((1,), 0.25, device="cuda")
    plan = ops.AdamW(ctx, tensors)
    seed, step, first = 0x123456789ABCDEF0, 7, 0
    plan.step(**HYPER, step=step, grad_scale=scale, seed=seed)
    plan.read_state()
    torch.cuda.synchronize()
    for n, t, o in zip(sizes, tensors, old):
        blocks = -(-n // BLOCK)
        g = _f64(o["grad"]) * 0.25
        if state == 32:
            m, v = _f64(o["m"]), _f64(o["v"])
        else:
            m = _decode(o["m"].cpu().numpy(), o["m_exp"].cpu().numpy(), 15)
            v = _decode(o["v"].cpu().numpy(), o["v_exp"].cpu().numpy(), 31)
        wd = t["weight_decay"]
        p1, m1, v1, u = _exact(_f64(o["p"]), g, m, v, wd, step)
        tol_m = 4 * EPS24 * (0.9 * np.abs(m) + 0.1 * np.abs(g))
        tol_v = 5 * EPS24 * (0.999 * v + 0.001 * g * g)
        tol_p = EPS24 * (2 * np.abs(_f64(o["p"])) + 10 * np.abs(u)) + HYPER["lr"] * 30 * np.divide(
            tol_m, np.sqrt(v1), out=np.zeros_like(v1), where=v1 > 0)
        assert (np.abs(_f64(t["p"]) - p1) <= tol_p).all()
        if "copy" in t:
            assert torch.equal(t["copy"], t["p"].to(t["copy"].dtype))
        if state == 32:
            assert (np.abs(_f64(t["m"]) - m1) <= tol_m).all() and (np.abs(_f64(t["v"]) - v1) <= tol_v).all()
        elif n:
            rm, rv = _random_bits(first * BLOCK + np.arange(n), seed)
            _codes_fit(t["m"].cpu().numpy(), t["m_exp"].cpu().numpy(), m1, 15, rm, tol_m)
            _codes_fit(t["v"].cpu().numpy(), t["v_exp"].cpu().numpy(), v1, 31, rv, tol_v)
            for name, top in (("m", 15), ("v", 31)):
                want = _decode(t[name].cpu().numpy(), t[name + "_exp"].cpu().numpy(), top)
                assert (_f64(t[name + "_seen"]) == want).all()
        first += blocks
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("state", [32, 8])
def test_first_step_from_cleared_state(harp, state):
    """m = v = 0 (zero bytes for 8 bits): the first step moves every weight by lr against its gradient's sign."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    t = _tensor(torch, 5000, state, torch.float32, None, 3, zero=True)
    t["grad"][17] = 0
    p = t["p"].clone()
    ops.AdamW(ctx, [t]).step(**HYPER, step=1, seed=5)
    want = p - HYPER["lr"] * torch.sign(t["grad"])
    want[17] = p[17]
    # |g| / (|g| + eps) for gradients of about 0.01, the smallest of 5,000 about 1e-6: within 1 % of one
    assert (t["p"] - want).abs().max().item() <= 0.011 * HYPER["lr"] + 4 * 2.0 ** -24 * 5
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("state", [32, 8])
def test_skip_leaves_everything(harp, state):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    t = _tensor(torch, 5000, state, torch.bfloat16, torch.bfloat16, 4)
    old = {k: x.clone() for k, x in t.items()}
    plan = ops.AdamW(ctx, [t])
    plan.step(**HYPER, step=2, skip=torch.ones(1, dtype=torch.int32, device="cuda"))
    assert all(torch.equal(t[k], old[k]) for k in old)
    plan.step(**HYPER, step=2, skip=torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert not torch.equal(t["p"], old["p"])
    ctx.close()


@pytest.mark.gpu
def test_infinities_and_nan_stay_with_their_elements_or_block(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    a, b = (_tensor(torch, 1000, s, torch.float32, None, 6) for s in (32, 8))
    for t in (a, b):
        t["grad"][300], t["grad"][700] = math.inf, math.nan
    plan = ops.AdamW(ctx, [a, b])
    plan.step(**HYPER, step=3)
    plan.read_state()
    hit = torch.zeros(1000, dtype=torch.bool, device="cuda")
    hit[300] = hit[700] = True
    for t in (a, b):
        assert torch.equal(torch.isfinite(t["p"]), ~hit)
    assert torch.equal(torch.isfinite(a["m"]), ~hit)
    block = torch.arange(1000, device="cuda") // BLOCK
    lost = (block == 1) | (block == 2)
    assert torch.equal(torch.isnan(b["m_seen"]), lost) and torch.equal(torch.isnan(b["v_seen"]), lost)
    ctx.close()


@pytest.mark.gpu
def test_rounding_to_8_bits_is_right_on_average(harp):
    """beta2 = 0.999 and gradients whose squares are half of v: every step takes 0.05 % off v, far below half a
    step of an 8-bit code (3 % to 6 %).  After 200 steps the mean over 16,384 elements is the exact average's."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    n = 16384
    t = _tensor(torch, n, 8, torch.float32, None, 8, zero=True)
    t["v"].fill_(30 * 8 + 4)               # 1.5 2^(E - 128) in blocks of exponent 127
    t["v_exp"].fill_(127)
    v0 = 0.75
    t["grad"].fill_(math.sqrt(v0 / 2))
    plan = ops.AdamW(ctx, [t])
    for k in range(200):
        plan.step(**HYPER, step=k + 1, seed=1000 + k)
    plan.read_state()
    got = _f64(t["v_seen"])
    want = v0 / 2 + v0 / 2 * 0.999 ** 200
    # each step's rounding has a variance of at most step size times what the step takes off, 1/16 * 0.00038 per step
    # (1/8 of 0.5 is the step): 200 of them, 16,384 independent elements, five deviations
    assert abs(got.mean() - want) <= 5 * math.sqrt(200 * 0.000375 / 16 / n)
    assert np.unique(got).size > 1
    ctx.close()


@pytest.mark.gpu
def test_the_same_bits_every_time_and_on_another_stream(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    runs = []
    for stream in (None, torch.cuda.Stream()):
        tensors = [_tensor(torch, n, s, torch.bfloat16, torch.bfloat16, 9 + n) for n, s in ((70_001, 32), (70_001, 8))]
        torch.cuda.synchronize()
        plan = ops.AdamW(ctx, tensors, stream=stream)
        for k in range(3):
            plan.step(**HYPER, step=k + 1, seed=k, stream=stream)
        torch.cuda.synchronize()
        runs.append(tensors)
    for a, b in zip(*runs):
        assert all(torch.equal(a[k], b[k]) for k in a)
    ctx.close()


@pytest.mark.gpu
def test_refusals(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    t = _tensor(torch, 100, 32, torch.float32, None, 1)
    e = _tensor(torch, 600, 8, torch.float32, None, 1)
    bad = [dict(t, p=t["p"][:99]), dict(t, m=t["m"].double()), dict(t, grad=t["grad"].double()),
           dict(t, copy=torch.zeros(100, device="cuda")), dict(t, weight_decay=-1.0), dict(t, weight_decay=math.inf),
           dict(e, m_exp=e["m_exp"][:2]), {k: x for k, x in e.items() if k != "v_exp"}, dict(t, unknown=1),
           {"p": t["p"]}, dict(t, p=t["p"].cpu()), dict(t, v=torch.zeros(200, device="cuda")[::2])]
    for entry in bad:
        with pytest.raises(harp.HarpError):
            ops.AdamW(ctx, [entry])
    plan = ops.AdamW(ctx, [t])
    for change in (dict(lr=-1.0), dict(lr=math.nan), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=math.inf), dict(step=0)):
        with pytest.raises(harp.HarpError) as err:
            plan.step(**dict(HYPER, step=1) | change)
        assert err.value.code == harp.ERR_INVALID_ARG
    ops.AdamW(ctx, []).step(**HYPER, step=1)          # nothing to do is no fault
    ctx.close()


def test_plan_bytes_refuses_malformed_entries():
    import ctypes
    from paper_2509_24859_amd import binding, operators as ops
    lib = binding.load_library()
    good = dict(n=1000, state=32, grad_type=ops.BF16, p=4096, grad=4096, m=4096, v=4096)

    def size(n_tensors=1, **kw):
        return lib.harp_adamw_plan_bytes(ctypes.byref(ops.harp_adamw_tensor(**dict(good, **kw))), n_tensors)

    assert size() > 0 and lib.harp_adamw_plan_bytes(None, 0) > 0
    for bad in (dict(n=-1), dict(n=1 << 40), dict(state=16), dict(grad_type=7), dict(p=0), dict(grad=0), dict(m=None), dict(v=None),
                dict(flags=1), dict(state=8), dict(p=4098), dict(grad=4097), dict(copy=4096, copy_type=0), dict(weight_decay=-0.1),
                dict(n_tensors=-1)):
        assert size(**bad) == 0, bad
    assert lib.harp_adamw_plan_bytes(None, 1) == 0
    assert lib.harp_adamw_plan(None, None, 0, None, 0, None, None) == binding.ERR_INVALID_ARG
    assert lib.harp_adamw_step(None, None, None, None) == binding.ERR_INVALID_ARG
    assert lib.harp_adamw_read_state(None, None, None) == binding.ERR_INVALID_ARG
