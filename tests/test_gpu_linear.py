"""The product with a fused epilogue and its gradients against their formulas in 64 bits.

Tolerances.  A product of two 16-bit values is exact in 32 bits.  A sum of R of them is off by at most R roundings of
2^-24 of the sum of magnitudes; in units of that, 64 + R / 8 is room for any order of a sum whose terms go in eight or
more at a time, and the sizes here are such that a wrong, missing or doubled term is far outside of it (the terms are
of order one, the room is a few millionths of their sum).  Activations and slopes are within 16 roundings of their
argument's magnitude, and change by at most 1.2 (slopes: 1.7) times what Z is off by.  A stored 16-bit result adds half
a unit of its own last place (2^-8 or 2^-11 of it).
"""
import math

import numpy as np
import pytest

EPS24 = 2.0 ** -24
UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _erf(z):
    return np.vectorize(math.erf, otypes=[float])(z) if z.size else z


def _act(z, act):
    """Activation and slope."""
    if act == "relu":
        return np.maximum(z, 0), (z > 0).astype(float)
    if act == "gelu":
        cdf = 0.5 * (1 + _erf(z / math.sqrt(2)))
        return z * cdf, cdf + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        th = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1 + th), 0.5 * (1 + th) + 0.5 * z * (1 - th ** 2) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1 / (1 + np.exp(-z))
        return z * s, s + z * s * (1 - s)
    return z, np.ones_like(z)


def _draw(rng, shape, kind, std=1.0):
    """Values of the type, in 64 bits."""
    import torch
    return torch.from_numpy(rng.standard_normal(shape) * std).to(kind).double().numpy()


def _gpu(a, kind, lead=0, pad=0):
    """On the GPU, `pad` columns wider and `lead` elements into its buffer; what is between holds NaN."""
    import torch
    if a is None:
        return None
    if a.ndim == 1:
        return torch.from_numpy(a).to(kind).cuda()
    rows, cols = a.shape
    buf = torch.full((lead + rows * (cols + pad) + 1,), float("nan"), dtype=kind, device="cuda")
    view = buf[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.from_numpy(a).to(kind))
    return view


def _host(t):
    return t.double().cpu().numpy()


def _within(got, want, room, unit, what):
    off, room = np.abs(got - want), room + unit * (np.abs(want) + room) + (2.0 ** -25 if unit == 2.0 ** -11 else 0)
    assert np.isfinite(got).all() and (off <= room).all(), (what, np.unravel_index(np.argmax(off - room), off.shape),
                                                            float((off / np.maximum(room, 1e-300)).max()))


# tokens, inputs, outputs: one token and long batches, sizes around every power of two that a tile may have, odd ones
SIZES = [(1, 1, 1), (1, 64, 128), (1, 4096, 512), (2, 1000, 1037), (3, 7, 5), (7, 1024, 264), (16, 520, 1024), (17, 2048, 96),
         (31, 33, 65), (32, 256, 256), (33, 264, 136), (64, 64, 64), (65, 8, 72), (100, 1000, 1000), (128, 128, 128), (129, 1152, 130),
         (200, 72, 1096), (255, 511, 257), (256, 256, 512), (257, 2056, 264), (300, 4104, 40), (513, 1224, 1000), (777, 320, 328),
         (1024, 512, 768)]
LAYOUTS = [dict(), dict(lead=1), dict(pad=8), dict(pad=1), dict(lead=8, pad=3)]


def _run(harp, case, direction):
    """(inputs, results, magnitudes) of one call."""
    import torch
    from paper_2509_24859_amd import operators as ops
    (m, k, n), kind, act, layout = case["size"], getattr(torch, case["type"]), case["act"], case["layout"]
    rng = np.random.default_rng(m * 7919 + k * 31 + n)
    ctx = harp.Context(0)
    ws = ops.linear_workspace(ctx, m, n, k)
    ws.fill_(0xFF)                                        # nothing may be taken from it
    put = lambda a: _gpu(a, kind, **layout)  # noqa: E731
    w = _draw(rng, (n, k), kind, k ** -0.5)
    v, out = {"w": w}, {}
    if direction == "forward":
        v["x"] = _draw(rng, (m, k), kind)
        v["bias"] = _draw(rng, (n,), kind) if case["bias"] else None
        v["residual"] = _draw(rng, (m, n), kind) if case["residual"] else None
        y, z = put(np.full((m, n), -7.0)), put(np.full((m, n), -7.0)) if case["save"] else None
        ops.harp_linear_forward(ctx, put(v["x"]), put(w), y, bias=_gpu(v["bias"], kind), act=act, residual=put(v["residual"]), z=z,
                                workspace=ws)
        out = {"y": y, "z": z}
    elif direction == "input":
        v["dy"] = _draw(rng, (m, n), kind)
        v["z"] = _draw(rng, (m, k), kind, 2.0) if act != "none" else None
        v["residual"] = _draw(rng, (m, k), kind) if case["residual"] else None
        out["dx"] = put(np.full((m, k), -7.0))
        ops.harp_linear_grad_input(ctx, put(v["dy"]), put(w), out["dx"], act=act, z=put(v["z"]), residual=put(v["residual"]), workspace=ws)
    else:
        v["dy"], v["x"] = _draw(rng, (m, n), kind), _draw(rng, (m, k), kind)
        wide = torch.float32 if case["wide"] else kind
        v["dw"], v["dbias"] = _draw(rng, (n, k), wide), _draw(rng, (n,), torch.float32)
        out = {"dw": _gpu(v["dw"], wide, **layout), "dbias": _gpu(v["dbias"], torch.float32) if case["bias"] else None}
        ops.harp_linear_grad_weight(ctx, put(v["dy"]), put(v["x"]), out["dw"], dbias=out["dbias"], accumulate=case["accumulate"], workspace=ws)
    torch.cuda.synchronize()
    ctx.close()
    return v, {a: _host(t) for a, t in out.items() if t is not None}


def _check(case, direction, v, got):
    (m, k, n), unit = case["size"], UNIT[case["type"]]
    if direction == "forward":
        z, mag = v["x"] @ v["w"].T, np.abs(v["x"]) @ np.abs(v["w"]).T
        if v["bias"] is not None:
            z, mag = z + v["bias"], mag + np.abs(v["bias"])
        off = (64 + k / 8) * EPS24 * mag
        y = _act(z, case["act"])[0]
        room = 1.2 * off + 16 * EPS24 * np.abs(z)
        if v["residual"] is not None:
            y, room = y + v["residual"], room + EPS24 * np.abs(v["residual"])
        if "z" in got:
            _within(got["z"], z, off, unit, "z")
        _within(got["y"], y, room, unit, "y")
    elif direction == "input":
        d, mag = v["dy"] @ v["w"], np.abs(v["dy"]) @ np.abs(v["w"])
        room = (64 + n / 8) * EPS24 * mag
        if v["z"] is not None:
            s = _act(v["z"], case["act"])[1]
            d, room = d * s, room * np.abs(s) + np.abs(d) * 32 * EPS24 * (1 + np.abs(v["z"]))
        if v["residual"] is not None:
            d, room = d + v["residual"], room + EPS24 * np.abs(v["residual"])
        _within(got["dx"], d, room, unit, "dx")
    else:
        d, mag = v["dy"].T @ v["x"], np.abs(v["dy"]).T @ np.abs(v["x"])
        b, b_mag = v["dy"].sum(0), np.abs(v["dy"]).sum(0)
        if case["accumulate"]:
            d, mag, b, b_mag = d + v["dw"], mag + np.abs(v["dw"]), b + v["dbias"], b_mag + np.abs(v["dbias"])
        _within(got["dw"], d, (64 + m / 8) * EPS24 * mag, UNIT["float32" if case["wide"] else case["type"]], "dw")
        if "dbias" in got:
            _within(got["dbias"], b, (64 + m / 8) * EPS24 * b_mag, 0.0, "dbias")


def _cases():
    """Every size in both types, the options dealt over them."""
    i, out = 0, []
    for size in SIZES:
        for kind in ("bfloat16", "float16"):
            i += 1
            out.append(dict(size=size, type=kind, act=ACTS[i % 5], bias=i % 2 == 0, residual=i % 3 == 0, save=i % 4 == 0,
                            accumulate=i % 3 == 1, wide=i % 4 < 2, layout=LAYOUTS[0]))
    for j, layout in enumerate(LAYOUTS[1:]):
        for size in ((1, 520, 136), (40, 264, 392), (300, 520, 264)):
            i += 1
            out.append(dict(size=size, type=("bfloat16", "float16")[i % 2], act=ACTS[i % 5], bias=True, residual=True, save=True,
                            accumulate=i % 2 == 0, wide=i % 3 == 0, layout=layout))
    return out


def _name(c):
    return "%s-%s-%s-%s" % ("x".join(map(str, c["size"])), c["type"], c["act"], "".join("%s%d" % x for x in c["layout"].items()))


@pytest.mark.gpu
@pytest.mark.parametrize("direction", ["forward", "input", "weight"])
@pytest.mark.parametrize("case", _cases(), ids=_name)
def test_a_product_is_the_formula(harp, case, direction):
    print(_name(case), direction, flush=True)
    v, got = _run(harp, case, direction)
    _check(case, direction, v, got)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [
    dict(size=(2048, 1024, 4096), type="bfloat16", act="gelu_tanh"), dict(size=(1537, 4904, 1224), type="float16", act="silu"),
    dict(size=(16, 8192, 4096), type="bfloat16", act="none"), dict(size=(4096, 264, 520), type="float16", act="relu"),
    dict(size=(24, 1024, 8192), type="bfloat16", act="gelu")], ids=lambda c: "x".join(map(str, c["size"])))
def test_larger_products_in_all_directions(harp, case):
    """Compared on the GPU, in 64 bits."""
    import torch
    from paper_2509_24859_amd import operators as ops
    (m, k, n), kind = case["size"], getattr(torch, case["type"])
    ctx = harp.Context(0)
    ws = ops.linear_workspace(ctx, m, n, k)
    x, w, dy = torch.randn(m, k, device="cuda").to(kind), (torch.randn(n, k, device="cuda") * k ** -0.5).to(kind), torch.randn(m, n, device="cuda").to(kind)
    zk = torch.randn(m, k, device="cuda").to(kind)
    y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
    ops.harp_linear_forward(ctx, x, w, y, act=case["act"], workspace=ws)
    ops.harp_linear_grad_input(ctx, dy, w, dx, act=case["act"], z=zk, workspace=ws)
    ops.harp_linear_grad_weight(ctx, dy, x, dw, dbias=db, workspace=ws)
    X, W, D = x.double(), w.double(), dy.double()
    unit = UNIT[case["type"]]
    z = X @ W.t()
    a, s = (torch.from_numpy(f) for f in _act(z.cpu().numpy(), case["act"]))
    room = (64 + k / 8) * EPS24 * (X.abs() @ W.t().abs())
    for name, got, want, room, u in (
            ("y", y, a.cuda(), 1.2 * room + 16 * EPS24 * z.abs(), unit),
            ("dx", dx, (D @ W) * torch.from_numpy(_act(_host(zk), case["act"])[1]).cuda(),
             (64 + n / 8) * EPS24 * (D.abs() @ W.abs()) * 1.2 + 32 * EPS24 * (D @ W).abs() * (1 + zk.double().abs()), unit),
            ("dw", dw, D.t() @ X, (64 + m / 8) * EPS24 * (D.abs().t() @ X.abs()), UNIT["float32"]),
            ("db", db, D.sum(0), (64 + m / 8) * EPS24 * D.abs().sum(0), 0.0)):
        off = (got.double() - want).abs()
        room = room + u * (want.abs() + room) + (2.0 ** -25 if u == 2.0 ** -11 else 0)
        assert (off <= room).all(), (name, (off / room).max().item())
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_slope_of_an_activation_alone(harp, act, kind):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    t = getattr(torch, kind)
    rng = np.random.default_rng(3)
    z, dy = _draw(rng, (37, 301), t, 3.0), _draw(rng, (37, 301), t)
    z[0, :4] = (0.0, -0.0, 30.0, -30.0)
    out = _gpu(np.zeros((37, 301)), t, 0, 3)
    ops.harp_act_grad(ctx, _gpu(dy, t, 1), _gpu(z, t, 0, 1), out, act)
    s = _act(z, act)[1]
    _within(_host(out), dy * s, np.abs(dy) * 32 * EPS24 * (1 + np.abs(z)), UNIT[kind], "dz")
    inplace = _gpu(dy, t)
    ops.harp_act_grad(ctx, inplace, _gpu(z, t), inplace, act)
    assert torch.equal(inplace, out)
    ctx.close()


@pytest.mark.parametrize("act", ACTS)
def test_the_slopes_against_differences(act):
    z = np.linspace(-6, 6, 1001) + 0.0005
    step = 1e-6
    numeric = (_act(z + step, act)[0] - _act(z - step, act)[0]) / (2 * step)
    assert np.abs(numeric - _act(z, act)[1]).max() < 1e-8


@pytest.mark.gpu
def test_masked_infinities_and_nan_go_where_the_formula_takes_them(harp):
    """A token of NaN, and a weight's row with an infinity, touch their own outputs alone."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    for m in (1, 20, 300):
        x, w = torch.rand(m, 200, device="cuda").bfloat16() + 1, torch.rand(264, 200, device="cuda").bfloat16()
        x[m - 1], w[17, 199] = math.nan, math.inf
        y = torch.empty(m, 264, device="cuda", dtype=torch.bfloat16)
        ops.harp_linear_forward(ctx, x, w, y, workspace=ops.linear_workspace(ctx, m, 264, 200))
        assert torch.isnan(y[m - 1]).all()
        if m > 1:
            assert torch.isposinf(y[:m - 1, 17]).all()
            rest = torch.cat((y[:m - 1, :17], y[:m - 1, 18:]), 1)
            assert torch.isfinite(rest).all()
    ctx.close()


@pytest.mark.gpu
def test_residual_in_place_graph_replays_and_other_streams(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    for m, k, n in ((1, 1024, 512), (20, 2048, 264), (300, 520, 264), (700, 1001, 1003)):
        ws = ops.linear_workspace(ctx, m, n, k)
        x, w, dy = torch.randn(m, k, device="cuda").half(), torch.randn(n, k, device="cuda").half() * k ** -0.5, torch.randn(m, n, device="cuda").half()
        r = torch.randn(m, n, device="cuda").half()
        y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty(n, device="cuda")

        def step(stream=None):
            ops.harp_linear_forward(ctx, x, w, y, residual=r, workspace=ws, stream=stream)
            ops.harp_linear_grad_input(ctx, dy, w, dx, residual=x, workspace=ws, stream=stream)
            ops.harp_linear_grad_weight(ctx, dy, x, dw, dbias=db, workspace=ws, stream=stream)

        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dx, dw, db)]
        over = r.clone()
        ops.harp_linear_forward(ctx, x, w, over, residual=over, workspace=ws)
        assert torch.equal(over, y)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        step(side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, dw, db)))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(3):
            for t in (y, dx, dw, db):
                t.fill_(-1)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, dw, db)))
    ctx.close()


@pytest.mark.gpu
def test_no_tokens(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    e, w = torch.empty(0, 64, device="cuda").half(), torch.randn(32, 64, device="cuda").half()
    ey, dw, db = torch.empty(0, 32, device="cuda").half(), torch.ones(32, 64, device="cuda"), torch.ones(32, device="cuda")
    ws = ops.linear_workspace(ctx, 0, 32, 64)
    ops.harp_linear_forward(ctx, e, w, ey, workspace=ws)
    ops.harp_linear_grad_input(ctx, ey, w, e, workspace=ws)
    ops.harp_linear_grad_weight(ctx, ey, e, dw, dbias=db, accumulate=True, workspace=ws)
    assert (dw == 1).all() and (db == 1).all()
    ops.harp_linear_grad_weight(ctx, ey, e, dw, dbias=db, workspace=ws)
    assert (dw == 0).all() and (db == 0).all()
    ctx.close()


@pytest.mark.gpu
def test_refusals(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    x, w, y = (torch.zeros(s, device="cuda", dtype=torch.bfloat16) for s in ((4, 64), (32, 64), (4, 32)))
    ws = ops.linear_workspace(ctx, 4, 32, 64)
    for a, k in (((x, w, y), dict(workspace=None)), ((x, w, y), dict(workspace=ws[:0])), ((x, w, y), dict(workspace=ws[1:])),
                 ((x.float(), w.float(), y.float()), {}), ((x, w.half(), y), {}), ((x, w[:, :63], y), {}), ((x, w, y[:3]), {}),
                 ((x, w, y), dict(act="tanh")), ((x, w, y), dict(act=9)), ((x, w, y), dict(bias=y[0].float())),
                 ((x, w, y), dict(bias=y[0][:31])), ((x, w, y), dict(z=x)), ((x.t().contiguous().t(), w, y), {}),
                 ((x.cpu(), w, y), {}), ((x[0], w, y), {})):
        with pytest.raises(harp.HarpError):
            ops.harp_linear_forward(ctx, *a, **dict(dict(workspace=ws), **k))
    for a, k in (((y, w, x), dict(act="relu")), ((y, w, w), {}), ((y, w, x), dict(residual=y))):
        with pytest.raises(harp.HarpError):
            ops.harp_linear_grad_input(ctx, *a, **dict(dict(workspace=ws), **k))
    for a, k in (((y, x, w.half()), {}), ((y, x, x), {}), ((y, x, w), dict(dbias=y[0]))):
        with pytest.raises(harp.HarpError):
            ops.harp_linear_grad_weight(ctx, *a, **dict(dict(workspace=ws), **k))
    with pytest.raises(harp.HarpError):
        ops.linear_workspace(ctx, 4, 0, 64)
    with pytest.raises(harp.HarpError):
        ops.linear_workspace(ctx, 1 << 31, 8, 64)
    ctx.close()


def test_null_contexts_are_refused_without_touching_the_gpu():
    from paper_2509_24859_amd import binding
    lib = binding.load_library()
    assert lib.harp_linear_workspace_bytes(None, 1, 1, 1) == 0
    for call in (lib.harp_linear_forward, lib.harp_linear_grad_input, lib.harp_linear_grad_weight):
        assert call(None, None, None, 0, None) == binding.ERR_INVALID_ARG
    assert lib.harp_act_grad(None, 1, 1, 0, 0, None, 1, None, 1, None, 1, None) == binding.ERR_INVALID_ARG
    assert lib.harp_norm_forward(None, None, None, 0, None, 0, None, 0, None, 0, None) == binding.ERR_INVALID_ARG
    assert lib.harp_norm_backward(None, None, None, None, 0, None) == binding.ERR_INVALID_ARG
    assert lib.harp_norm_workspace_bytes(None, None) == 0
