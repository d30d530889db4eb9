"""The gated block and the way back through it against their formulas in 64 bits.

Tolerances.  Z and dH are sums of R products of 16-bit values, exact in 32 bits each: off by at most (64 + R / 8) 2^-24 of the sum of
magnitudes (terms go in eight or more at a time).  Activations are within 16 roundings of their argument's magnitude, slopes within 32 of it and one,
and change by at most 1.2 (slopes: 1.7) times what Z is off by; each further product adds one rounding.  A stored result adds
half a unit of its last place, 2^-8 or 2^-11 of it, in float16 at least 2^-25.
"""
import math

import numpy as np
import pytest

from operator_context import HostContext, refused
from test_gpu_linear import EPS24, UNIT, _act, _draw, _gpu, _host, _within

# tokens, channels, width: few tokens and many, around the tiles' sides, odd ones, sums that are shared out
SIZES = [(1, 1, 1), (1, 64, 128), (1, 4096, 264), (3, 7, 5), (7, 1000, 1037), (16, 520, 512), (17, 2048, 96), (32, 256, 33), (33, 264, 136),
         (64, 64, 64), (65, 8, 72), (100, 1000, 1000), (128, 128, 64), (129, 4104, 130), (200, 72, 1096), (255, 511, 257), (256, 256, 128),
         (257, 2056, 264), (513, 1224, 1000), (1024, 512, 768), (2100, 320, 4100)]
LAYOUTS = [dict(), dict(lead=1), dict(pad=8), dict(pad=1), dict(lead=8, pad=3)]
ACTS = ("silu", "gelu_tanh", "gelu", "relu", "none")
CASES = [dict(size=s, type=t, act=ACTS[(i + j) % 5], layout=LAYOUTS[(i + 2 * j) % 5], more=(i + j) % 2 == 0)
         for i, s in enumerate(SIZES) for j, t in enumerate(("bfloat16", "float16"))]


def _id(c):
    return "%dx%dx%d-%s-%s-%s" % (*c["size"], c["type"], c["act"], "".join("%s%d" % x for x in c["layout"].items()))


def _forward(harp, c, rng):
    import torch
    from paper_2509_24859_amd import operators as ops
    (m, k, f), kind = c["size"], getattr(torch, c["type"])
    ctx = harp.Context(0)
    ws = ops.gated_workspace(ctx, m, f, k)
    ws.fill_(0xFF)                                        # nothing may be taken from it
    x, w = _draw(rng, (m, k), kind), _draw(rng, (2 * f, k), kind, k ** -0.5)
    bias = _draw(rng, (2 * f,), kind) if c["more"] else None
    put = lambda a: _gpu(a, kind, **c["layout"])  # noqa: E731
    h, z = put(np.full((m, f), -7.0)), put(np.full((m, 2 * f), -7.0)) if c["more"] else None
    call = lambda: ops.harp_gated_forward(ctx, put(x), put(w), h, bias=_gpu(bias, kind), act=c["act"], z=z, workspace=ws)  # noqa: E731
    call()
    return ctx, x, w, bias, h, z


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=_id)
def test_forward(harp, case):
    rng = np.random.default_rng(sum(case["size"]))
    ctx, x, w, bias, h, z = _forward(harp, case, rng)
    (_, k, f), unit = case["size"], UNIT[case["type"]]
    want, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        want, mag = want + bias, mag + np.abs(bias)
    room = (64 + k / 8) * EPS24 * mag
    if z is not None:
        _within(_host(z), want, room, unit, "z")
    a, _ = _act(want[:, :f], case["act"])
    off = 1.2 * room[:, :f] + 16 * EPS24 * np.abs(want[:, :f])
    up, off_up = want[:, f:], room[:, f:]
    _within(_host(h), a * up, off * (np.abs(up) + off_up) + np.abs(a) * off_up + 2 * EPS24 * np.abs(a * up), unit, "h")
    ctx.close()


def _back_want(dh, room, z, act):
    """(dz, its room, h, its room)."""
    f = z.shape[1] // 2
    gate, up = z[:, :f], z[:, f:]
    a, s = _act(gate, act)
    off = 16 * EPS24 * np.abs(gate)
    dg, du = dh * up * s, dh * a
    rg = (room * np.abs(s) + (np.abs(dh) + room) * 32 * EPS24 * (1 + np.abs(gate))) * np.abs(up) + 4 * EPS24 * np.abs(dg)
    ru = room * np.abs(a) + (np.abs(dh) + room) * off + 4 * EPS24 * np.abs(du)
    return np.concatenate((dg, du), 1), np.concatenate((rg, ru), 1), a * up, off * np.abs(up) + 2 * EPS24 * np.abs(a * up)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=_id)
def test_back(harp, case):
    import torch
    from paper_2509_24859_amd import operators as ops
    (m, n, f), kind, unit = case["size"], getattr(torch, case["type"]), UNIT[case["type"]]
    rng = np.random.default_rng(sum(case["size"]) + 1)
    ctx = harp.Context(0)
    ws = ops.gated_workspace(ctx, m, f, n)
    ws.fill_(0xFF)
    put = lambda a: _gpu(a, kind, **case["layout"])  # noqa: E731
    dy, w, z = _draw(rng, (m, n), kind), _draw(rng, (n, f), kind, n ** -0.5), _draw(rng, (m, 2 * f), kind, 2.0)
    dz, h = put(np.full((m, 2 * f), -7.0)), put(np.full((m, f), -7.0)) if case["more"] else None
    ops.harp_gated_grad(ctx, put(dy), put(w), put(z), dz, act=case["act"], h=h, workspace=ws)
    want, room, want_h, room_h = _back_want(dy @ w, (64 + n / 8) * EPS24 * (np.abs(dy) @ np.abs(w)), z, case["act"])
    _within(_host(dz), want, room, unit, "dz")
    if h is not None:
        _within(_host(h), want_h, room_h, unit, "h")
    # dH given instead of made, dZ in Z's place
    dh, zz = _draw(rng, (m, f), kind), put(z)
    want, room, _, _ = _back_want(dh, np.zeros_like(dh), z, case["act"])
    ops.harp_gated_grad(ctx, put(dh), None, zz, zz, act=case["act"])
    _within(_host(zz), want, room, unit, "dz of dh")
    ctx.close()


@pytest.mark.gpu
def test_dz_in_the_place_of_z(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    for m, n, f in ((300, 520, 600), (129, 4104, 130), (70, 64, 33)):
        dy, w, z = (torch.randn(s, device="cuda").bfloat16() for s in ((m, n), (n, f), (m, 2 * f)))
        ws = ops.gated_workspace(ctx, m, f, n)
        want = torch.empty_like(z)
        ops.harp_gated_grad(ctx, dy, w, z, want, workspace=ws)
        ops.harp_gated_grad(ctx, dy, w, z, z, workspace=ws)
        assert torch.equal(z, want)
    ctx.close()


@pytest.mark.gpu
def test_gradient_by_differences(harp):
    """d(sum of H g) along a direction of Z, from the formula in 64 bits on both sides of Z, against what the call gives for dH = g.
    The difference quotient's own error is the third derivative's step^2 / 6, under 1e-6 of the terms here; dZ is rounded to
    float16, and a sum of n terms of either sign gathers at most their sum of magnitudes times 2^-11."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    rng = np.random.default_rng(5)
    m, f, step = 20, 24, 1e-3
    z, g, way = _draw(rng, (m, 2 * f), torch.float16), _draw(rng, (m, f), torch.float16), rng.standard_normal((m, 2 * f))
    for act in ("silu", "gelu", "gelu_tanh", "none"):
        dz = torch.empty(m, 2 * f, dtype=torch.float16, device="cuda")
        ops.harp_gated_grad(ctx, _gpu(g, torch.float16), None, _gpu(z, torch.float16), dz, act=act)
        value = lambda at: (_act(at[:, :f], act)[0] * at[:, f:] * g).sum()  # noqa: E731
        slope = (value(z + step * way) - value(z - step * way)) / (2 * step)
        terms = _host(dz) * way
        assert abs(terms.sum() - slope) <= (2.0 ** -11 + 1e-5) * np.abs(terms).sum()
    ctx.close()


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_rows(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    for m in (8, 300):
        x, w = torch.randn(m, 264, device="cuda").bfloat16(), torch.randn(160, 264, device="cuda").bfloat16()
        x[2, 5], x[4, 100] = math.nan, math.inf
        h = torch.empty(m, 80, dtype=torch.bfloat16, device="cuda")
        ops.harp_gated_forward(ctx, x, w, h, workspace=ops.gated_workspace(ctx, m, 80, 264))
        bad = ~torch.isfinite(h).all(1)
        assert bad[2] and bad[4] and bad.sum() == 2
    ctx.close()


@pytest.mark.gpu
def test_streams_graphs_and_no_tokens(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    m, k, f = 150, 4104, 136                                  # sums are shared out: two launches
    x, w, w2 = (torch.randn(s, device="cuda").bfloat16() for s in ((m, k), (2 * f, k), (k, f)))
    dy = torch.randn(m, k, device="cuda").bfloat16()
    ws = ops.gated_workspace(ctx, m, f, k)
    b16 = dict(dtype=torch.bfloat16, device="cuda")
    h, z, dz, h2 = torch.empty(m, f, **b16), torch.empty(m, 2 * f, **b16), torch.empty(m, 2 * f, **b16), torch.empty(m, f, **b16)

    def both(stream=None):
        ops.harp_gated_forward(ctx, x, w, h, z=z, workspace=ws, stream=stream)
        ops.harp_gated_grad(ctx, dy, w2, z, dz, h=h2, workspace=ws, stream=stream)

    both()
    want = [t.clone() for t in (h, z, dz, h2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (h, z, dz, h2)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in (h, z, dz, h2):
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (h, z, dz, h2)))
    ops.harp_gated_forward(ctx, x[:0], w, h[:0], workspace=ws)
    ops.harp_gated_grad(ctx, dy[:0], w2, z[:0], dz[:0], workspace=ws)
    ctx.close()


@pytest.mark.gpu
def test_offsets_beyond_32_bits(harp):
    """Rows 2^22 elements and more apart, 600 of them."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    buf = torch.empty(600, (1 << 22) + 8, dtype=torch.bfloat16, device="cuda")
    m, k, f = 600, 136, 72
    x, h, z, dz = (buf[:, at:at + n] for at, n in ((0, k), (1000, f), (2000, 2 * f), (3000, 2 * f)))
    x.copy_(torch.randn(m, k, device="cuda"))
    w, w2, dy = (torch.randn(s, device="cuda").bfloat16() for s in ((2 * f, k), (k, f), (m, k)))
    ws = ops.gated_workspace(ctx, m, f, k)
    near = [torch.empty(m, n, dtype=torch.bfloat16, device="cuda") for n in (f, 2 * f, 2 * f)]
    ops.harp_gated_forward(ctx, x, w, h, z=z, workspace=ws)
    ops.harp_gated_forward(ctx, x.contiguous(), w, near[0], z=near[1], workspace=ws)
    ops.harp_gated_grad(ctx, dy, w2, z, dz, workspace=ws)
    ops.harp_gated_grad(ctx, dy, w2, near[1], near[2], workspace=ws)
    assert torch.equal(h, near[0]) and torch.equal(z, near[1]) and torch.equal(dz, near[2])
    ctx.close()


def test_refusals(monkeypatch):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = HostContext()
    b = torch.bfloat16
    x, w, h, z = torch.zeros(4, 8, dtype=b), torch.zeros(12, 8, dtype=b), torch.zeros(4, 6, dtype=b), torch.zeros(4, 12, dtype=b)
    # memory of the size that is asked for, not aligned or too small
    need = ops.gated_workspace(ctx, 4, 6, 8)
    off = 1 if need.data_ptr() % 256 == 0 else 0
    fwd = lambda *a, **k: refused(monkeypatch, ops.harp_gated_forward, ctx, *a, **k)  # noqa: E731
    for a, k in (((x.float(), w.float(), h.float()), {}), ((x, w[:11], h), {}), ((x, w[:, :7], h), {}), ((x, w, h[:, :5]), {}),
                 ((x, w, h), dict(z=h)), ((x, w, h), dict(bias=torch.zeros(6, dtype=b))), ((x, w, h), dict(act="swish")),
                 ((x, w, h), dict(act=9)), ((x[0], w, h), {}), ((x.half(), w, h), {}), ((x, w, h), dict(workspace=None)),
                 ((x, w, h), dict(workspace=need[off:])), ((x, w, h.t().contiguous().t()), {})):
        fwd(*a, **k)
    dy, w2 = torch.zeros(4, 8, dtype=b), torch.zeros(8, 6, dtype=b)
    for a, k in (((dy, w2[:7], z, z), {}), ((dy, None, z, z), {}), ((dy, w2, z[:, :11], z), {}), ((dy, w2, z, h), {}), ((dy, w2, z, z), dict(h=z)),
                 ((dy, w2, z, z), dict(workspace=None)), ((dy, w2, z, z), dict(act="swish"))):
        refused(monkeypatch, ops.harp_gated_grad, ctx, *a, **k)
    for sizes in ((-1, 6, 8), (1 << 31, 6, 8), (4, 0, 8), (4, 6, 0), (4, 1 << 21, 8), (4, 6, 1 << 21)):
        refused(monkeypatch, ops.gated_workspace, ctx, *sizes)


def test_gradient_over_z_at_other_distances_is_refused(monkeypatch):
    import torch
    from paper_2509_24859_amd import binding, operators as ops
    ctx, memory = HostContext(), torch.zeros(4, 16, dtype=torch.bfloat16)
    z, dz, dh = memory[:, :12], memory.view(-1)[:48].view(4, 12), torch.zeros(4, 6, dtype=torch.bfloat16)
    assert refused(monkeypatch, ops.harp_gated_grad, ctx, dh, None, z, dz) == binding.ERR_SHAPE
