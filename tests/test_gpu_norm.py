"""Norms around a block with gate and residual scale against their formulas in 64 bits.

Tolerances.  A sum over a row is at most 8 + 6 + 16 roundings deep (a thread's channels, a wavefront, the
wavefronts); with the quotient, the root and the products a norm is within 40 roundings of 2^-24 of the magnitudes that
flow into it, and the chain here is at most four such sums long (mean, square, and the same of the second norm): 160 in
the forward pass, 300 in the backward pass, whose gradients pass through both norms' statistics once more.  Sums over
rows add one rounding a row.  "Magnitudes" are the same formulas with every term taken by its absolute value.  A stored
16-bit result adds half a unit of its own last place (2^-8 or 2^-11 of it).
"""
import itertools
import math

import numpy as np
import pytest

EPS24 = 2.0 ** -24
UNIT = {"float32": 0.0, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
EPS = 1e-5


def _gate(g, act, rows, per):
    if g is None:
        return None, None
    f = 1 / (1 + np.exp(-g)) if act == "sigmoid" else g
    df = f * (1 - f) if act == "sigmoid" else np.ones_like(g)
    at = np.arange(rows) // per
    return f[at], df[at]


class _Norm:
    """One norm of rows: centered values, normalised values, and bounds on what rounding does to them."""

    def __init__(self, a, mag, kind, w, b):
        self.kind = kind
        self.w = np.ones(a.shape[1]) if w is None else w
        self.b = np.zeros(a.shape[1]) if b is None else b
        self.c = a - a.mean(1, keepdims=True) if kind == "layer" else a
        self.mag = mag + mag.mean(1, keepdims=True) if kind == "layer" else mag
        ms = (self.c ** 2).mean(1, keepdims=True) + EPS
        self.rstd = 1 / np.sqrt(ms)
        self.hat = self.c * self.rstd
        loss = (np.abs(self.c) * self.mag).mean(1, keepdims=True) / ms      # of rstd, relative
        self.hat_mag = self.mag * self.rstd + np.abs(self.hat) * (1 + loss)
        self.out = self.hat * self.w + self.b
        self.out_mag = self.hat_mag * np.abs(self.w) + np.abs(self.b)

    def back(self, d, d_mag):
        """Gradient of the input for d at the output (before the weight), and its magnitude."""
        m = lambda v: v.mean(1, keepdims=True)  # noqa: E731
        e = d - self.hat * m(d * self.hat)
        mag = d_mag + np.abs(self.hat) * m(d_mag * self.hat_mag) + self.hat_mag * m(np.abs(d) * self.hat_mag)
        if self.kind == "layer":
            e, mag = e - m(d), mag + m(d_mag)
        ratio = 1 + (self.hat_mag.max(1, keepdims=True) / np.maximum(np.abs(self.hat).max(1, keepdims=True), 1e-3))
        return e * self.rstd, mag * self.rstd * ratio


def _forward(c, v):
    rows = c["rows"]
    y = v["y"]
    if y is None:
        h, mag = v["x"], np.abs(v["x"])
        after = None
    else:
        after = None if c["after"] == "none" else _Norm(y, np.abs(y), c["after"], v["w_after"], v["b_after"])
        t, t_mag = (y, np.abs(y)) if after is None else (after.out, after.out_mag)
        f, _ = _gate(v["gate"], c["gate_act"], rows, c["per"])
        k = np.ones_like(t) if f is None else f
        k = k if v["scale"] is None else k * v["scale"]
        h, mag = k * t, np.abs(k) * t_mag
        if v["x"] is not None:
            h, mag = h + v["x"], mag + np.abs(v["x"])
    before = None if c["before"] == "none" else _Norm(h, mag, c["before"], v["w_before"], v["b_before"])
    return h, mag, before


def _backward(c, v):
    """{name: (value, magnitude)}; h is given, as the forward pass stored it."""
    rows, out = c["rows"], {}
    D, mag = (np.zeros_like(v["h"]),) * 2 if v["dh"] is None else (v["dh"], np.abs(v["dh"]))
    if v["dz"] is not None:
        n = _Norm(v["h"], np.abs(v["h"]), c["before"], v["w_before"], v["b_before"])
        e, m = n.back(v["dz"] * n.w, np.abs(v["dz"] * n.w))
        D, mag = D + e, mag + m
        out["dw_before"] = ((v["dz"] * n.hat).sum(0), (np.abs(v["dz"]) * n.hat_mag).sum(0))
        out["db_before"] = (v["dz"].sum(0), np.abs(v["dz"]).sum(0))
    out["dx"] = (D, mag)
    y = v["y"]
    if y is None:
        return out
    after = None if c["after"] == "none" else _Norm(y, np.abs(y), c["after"], v["w_after"], v["b_after"])
    t, t_mag = (y, np.abs(y)) if after is None else (after.out, after.out_mag)
    hat, hat_mag = (y, np.abs(y)) if after is None else (after.hat, after.hat_mag)
    f, df = _gate(v["gate"], c["gate_act"], rows, c["per"])
    sc = np.ones(y.shape[1]) if v["scale"] is None else v["scale"]
    fk = np.ones_like(y) if f is None else f
    out["dscale"] = ((D * t * fk).sum(0), (mag * t_mag * np.abs(fk)).sum(0))
    if f is not None:
        per, groups = c["per"], -(-rows // c["per"])
        each, each_mag = D * t * sc * df, mag * t_mag * np.abs(sc * df)
        out["dgate"] = tuple(np.stack([e[g * per:(g + 1) * per].sum(0) for g in range(groups)]) for e in (each, each_mag))
    dt, dt_mag = D * fk * sc, mag * np.abs(fk * sc)
    out["dw_after"] = ((dt * hat).sum(0), (dt_mag * hat_mag).sum(0))
    out["db_after"] = (dt.sum(0), dt_mag.sum(0))
    out["dy"] = (dt, dt_mag) if after is None else after.back(dt * after.w, dt_mag * np.abs(after.w))
    return out


def _values(c, rng):
    """Inputs in 64 bits, already rounded to the type that holds them."""
    import torch
    kind = getattr(torch, c["type"])

    def data(shape, std=1.0):
        return torch.from_numpy(rng.standard_normal(shape) * std).to(kind).double().numpy()

    def vector(mean, std):
        return (mean + std * rng.standard_normal(c["cols"])).astype(np.float32).astype(np.float64)

    rows, cols = c["rows"], c["cols"]
    v = {"x": data((rows, cols), 3.0), "y": data((rows, cols)), "h": data((rows, cols), 3.0), "dh": data((rows, cols), 0.1),
         "dz": data((rows, cols)), "gate": data((-(-rows // c["per"]), cols)) if c["per"] else None,
         "scale": vector(0, 0.5) if c["scale"] else None}
    for at in ("after", "before"):
        v["w_" + at] = vector(1, 0.2) if c[at] != "none" and c["weights"] else None
        v["b_" + at] = vector(0, 0.2) if c[at] != "none" and c["weights"] else None
    for name in c.get("without", ()):
        v[name] = None
    return v


def _on_gpu(a, dtype, lead=0, pad=0):
    """On the GPU, `pad` columns wider and `lead` elements into its buffer."""
    import torch
    if a is None:
        return None
    if a.ndim == 1:
        return torch.from_numpy(a).to(dtype).cuda()
    rows, cols = a.shape
    buf = torch.full((lead + rows * (cols + pad),), float("nan"), dtype=dtype, device="cuda")
    view = buf[lead:].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.from_numpy(a).to(dtype))
    return view


def _case(rows, cols, type="float32", after="rms", before="rms", per=0, gate_act="linear", scale=True, weights=True, **more):
    return dict(rows=rows, cols=cols, type=type, after=after, before=before, per=per, gate_act=gate_act, scale=scale,
                weights=weights, **more)


CASES = [
    _case(1, 1, "float32", "layer", "layer"), _case(3, 2), _case(1, 8192, "bfloat16"), _case(5, 8191, "float16", "layer", "rms"),
    _case(300, 64, "bfloat16", per=1, gate_act="sigmoid"), _case(300, 65, "float16", "layer", "layer", per=300),
    _case(600, 1000, "bfloat16", "rms", "layer", per=7), _case(257, 1155, "float32", "layer", "layer", per=100, gate_act="sigmoid", scale=False),
    _case(600, 2048, "bfloat16", "none", "rms", per=1000), _case(40, 4096, "float16", "none", "layer", scale=False, weights=False),
    _case(600, 136, "float32", "rms", "layer", per=599, weights=False), _case(1, 7, "float16", per=5),
    _case(90, 520, "bfloat16", "layer", "none"), _case(64, 512, "float32", "rms", "rms", per=8, pad=8),
    _case(64, 512, "bfloat16", "rms", "layer", per=8, pad=1), _case(64, 512, "float16", "layer", "rms", per=64, lead=1),
    _case(33, 1024, "bfloat16", without=("x",)), _case(33, 1024, "bfloat16", "none", "rms", without=("y",), scale=False),
    _case(33, 1000, "float32", "layer", "rms", without=("dh",)), _case(33, 1000, "float32", "layer", "rms", without=("dz",)),
]


def _run(harp, c, direction, seed=0):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    v = _values(c, np.random.default_rng(seed))
    kind = getattr(torch, c["type"])
    shape = dict(lead=c.get("lead", 0), pad=c.get("pad", 0))
    put = lambda n: _on_gpu(v[n], kind, **shape)  # noqa: E731
    vec = {n: _on_gpu(v[n], torch.float32) for n in ("scale", "w_after", "b_after", "w_before", "b_before")}
    form = dict(after=c["after"], before=c["before"], gate=put("gate"), rows_per_gate=c["per"] or 1, gate_act=c["gate_act"], eps=EPS, **vec)
    empty = lambda: _on_gpu(np.full((c["rows"], c["cols"]), -7.0), kind, **shape)  # noqa: E731
    if direction == "forward":
        h, z = empty(), empty() if c["before"] != "none" else None
        ops.harp_norm_forward(ctx, put("x"), put("y"), h, z, **form)
        got = {"h": h, "z": z}
    else:
        with_y = v["y"] is not None
        dx, dy = empty(), empty() if with_y else None
        dz = put("dz") if c["before"] != "none" else None
        grads = {n: torch.full((c["cols"],), -7.0, device="cuda") for n in ("dw_before", "db_before")
                 + (("dw_after", "db_after", "dscale") if with_y else ())}
        if v["gate"] is not None:
            grads["dgate"] = _on_gpu(np.full(v["gate"].shape, -7.0), kind, **shape)
        ops.harp_norm_backward(ctx, put("dh"), dz, put("h"), put("y"), dx, dy, **form, **grads,
                               workspace=ops.norm_workspace(ctx, c["rows"], c["cols"], c["per"]))
        got = dict(grads, dx=dx, dy=dy)
        if dz is None:
            v["dz"] = None
    torch.cuda.synchronize()
    got = {n: t.double().cpu().numpy() for n, t in got.items() if t is not None}
    ctx.close()
    return v, got


def _within(got, want, mag, count, unit, what):
    off = np.abs(got - want)
    room = count * EPS24 * mag + unit * np.abs(want) + (2.0 ** -25 if unit == 2.0 ** -11 else 0)
    worst = np.unravel_index(np.argmax(off - room), off.shape)
    assert (off <= room).all(), (what, worst, got[worst], want[worst], room[worst])


@pytest.mark.gpu
@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(str(x) for x in list(c.values())[:6]))
def test_forward_is_the_formula(harp, c):
    v, got = _run(harp, c, "forward")
    h, mag, before = _forward(c, v)
    unit = UNIT[c["type"]]
    if v["y"] is not None:
        _within(got["h"], h, mag, 160, unit, "h")
    if before is not None:
        _within(got["z"], before.out, before.out_mag, 160, unit, "z")


@pytest.mark.gpu
@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(str(x) for x in list(c.values())[:6]))
def test_backward_is_the_formula(harp, c):
    v, got = _run(harp, c, "backward")
    want = _backward(c, v)
    for name, value in got.items():
        if name not in want:                      # no dz: the sums of the norm before are zero
            assert name in ("dw_before", "db_before") and (value == 0).all(), name
            continue
        whole = name in ("dx", "dy", "dgate")
        count = 300 + (0 if name in ("dx", "dy") else c["rows"])
        _within(value, *want[name], count, UNIT[c["type"]] if whole else 0.0, name)


@pytest.mark.parametrize("kinds", itertools.product(("none", "rms", "layer"), ("rms", "layer")))
def test_the_formula_of_the_gradient_against_differences(kinds):
    """Central differences of the forward formula, in 64 bits: off by step^2 times a third derivative of order one,
    and by rounding over the step."""
    c = _case(4, 5, "float32", *kinds, per=3, gate_act="sigmoid")
    rng = np.random.default_rng(1)
    v = _values(c, rng)
    up = {"h": rng.standard_normal((4, 5)), "z": rng.standard_normal((4, 5))}

    def loss(v):
        h, _, before = _forward(c, v)
        return (h * up["h"]).sum() + (before.out * up["z"]).sum()

    v["h"] = _forward(c, v)[0]
    got = _backward(c, dict(v, dh=up["h"], dz=up["z"]))
    step = 1e-5
    for name, grad in (("x", "dx"), ("y", "dy"), ("gate", "dgate"), ("scale", "dscale"), ("w_after", "dw_after"),
                       ("b_after", "db_after"), ("w_before", "dw_before"), ("b_before", "db_before")):
        if v[name] is None:
            continue
        flat = np.zeros(v[name].size)
        for i in range(flat.size):
            for sign in (1, -1):
                moved = v[name].copy()
                moved.reshape(-1)[i] += sign * step
                flat[i] += sign * loss(dict(v, **{name: moved})) / (2 * step)
        assert np.abs(flat - got[grad][0].reshape(-1)).max() < 1e-7, name


@pytest.mark.gpu
def test_sums_are_added_to_when_asked(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    rows, cols = 100, 256
    t = [torch.randn(rows, cols, device="cuda") for _ in range(4)]
    ws = ops.norm_workspace(ctx, rows, cols)
    out = [torch.full((cols,), 2.0, device="cuda") for _ in range(2)]
    dx, dy = torch.empty_like(t[0]), torch.empty_like(t[0])
    ops.harp_norm_backward(ctx, t[0], t[1], t[2], t[3], dx, dy, dw_before=out[0], workspace=ws)
    ops.harp_norm_backward(ctx, t[0], t[1], t[2], t[3], dx, dy, dw_before=out[1], workspace=ws, accumulate=True)
    assert torch.equal(out[0] + 2.0, out[1])
    ctx.close()


@pytest.mark.gpu
def test_outputs_over_inputs_and_graph_replays(harp):
    """h over x, z over y; dx over dh, dy over y: the same bits as apart; and a captured pass replays to them."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    rows, cols = 300, 1032
    w = torch.rand(cols, device="cuda")
    gate = torch.randn(3, cols, device="cuda").bfloat16()
    x, y, dh, dz = (torch.randn(rows, cols, device="cuda").bfloat16() for _ in range(4))
    form = dict(after="rms", before="layer", gate=gate, rows_per_gate=100, w_after=w, w_before=w)
    h, z = torch.empty_like(x), torch.empty_like(x)
    ops.harp_norm_forward(ctx, x, y, h, z, **form)
    x2, y2 = x.clone(), y.clone()
    ops.harp_norm_forward(ctx, x2, y2, x2, y2, **form)
    assert torch.equal(x2, h) and torch.equal(y2, z)
    ws = ops.norm_workspace(ctx, rows, cols, 100)
    dx, dy, dg, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gate), torch.empty_like(w)

    def backward():
        ops.harp_norm_backward(ctx, dh, dz, h, y, dx, dy, **form, dgate=dg, dw_before=dw, workspace=ws)

    backward()
    want = [t.clone() for t in (dx, dy, dg, dw)]
    dh2, y3 = dh.clone(), y.clone()
    ops.harp_norm_backward(ctx, dh2, dz, h, y3, dh2, y3, **form, workspace=ws)
    assert torch.equal(dh2, want[0]) and torch.equal(y3, want[1])
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        backward()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        backward()
    for _ in range(3):
        for t in (dx, dy, dg, dw):
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (dx, dy, dg, dw)))
    ctx.close()


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_rows(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    x, y = torch.randn(8, 513, device="cuda"), torch.randn(8, 513, device="cuda")
    y[2, 5], x[4, 512] = math.nan, math.inf
    h, z = torch.empty_like(x), torch.empty_like(x)
    ops.harp_norm_forward(ctx, x, y, h, z)
    ok = torch.ones(8, dtype=torch.bool, device="cuda")
    ok[2] = ok[4] = False
    assert torch.equal(torch.isfinite(z).all(1), ok) and torch.isnan(z[2]).all()
    ctx.close()


@pytest.mark.gpu
def test_no_rows(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    e = torch.empty(0, 64, device="cuda")
    dw = torch.ones(64, device="cuda")
    ops.harp_norm_forward(ctx, e, e, e, e)
    for per in (0, 4):
        ws = ops.norm_workspace(ctx, 0, 64, per)
        kw = dict(gate=e, rows_per_gate=per) if per else {}
        ops.harp_norm_backward(ctx, e, e, e, e, e, e, dw_before=dw, workspace=ws, accumulate=True, **kw)
        assert (dw == 1).all()
    ops.harp_norm_backward(ctx, e, e, e, e, e, e, dw_before=dw, workspace=ws)
    assert (dw == 0).all()
    ctx.close()


@pytest.mark.gpu
def test_refusals(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    x, y, h, z = (torch.zeros(4, 64, device="cuda") for _ in range(4))
    w = torch.ones(64, device="cuda")
    fwd = lambda *a, **k: ops.harp_norm_forward(ctx, *a, **k)  # noqa: E731
    wide = torch.zeros(2, ops.NORM_MAX_COLS + 1, device="cuda")
    for a, k in (((x, y, h, None), {}), ((None, None, h, z), {}), ((x, None, h, None), dict(before="none")),
                 ((x, y[:3], h, z), {}), ((x, y.double(), h, z), {}), ((x, y.t().contiguous().t(), h, z), {}),
                 ((x, y, h, z), dict(w_after=w[:63])), ((x, y, h, z), dict(w_after=w.half())),
                 ((x, y, h, z), dict(gate=x, rows_per_gate=0)), ((x, y, h, z), dict(gate=x, rows_per_gate=2)),
                 ((x, y, h, z), dict(after="batch")), ((x, y, h, z), dict(after=3)), ((x, y, h, z), dict(eps=-1.0)),
                 ((x.cpu(), y, h, z), {}), ((wide, wide, wide, wide), {}), ((x.long(), y, h, z), {})):
        with pytest.raises(harp.HarpError):
            fwd(*a, **k)
    ws = ops.norm_workspace(ctx, 4, 64)
    bwd = lambda *a, **k: ops.harp_norm_backward(ctx, *a, **dict(dict(workspace=ws), **k))  # noqa: E731
    for a, k in (((None, None, h, y, x, z), {}), ((None, x, None, y, z, h), {}), ((x, None, h, None, z, h), {}),
                 ((x, z, h, y, z, h), dict(workspace=None)), ((x, z, h, y, z, h), dict(workspace=ws[:256])),
                 ((x, z, h, y, z, h), dict(workspace=ws[1:])), ((x, z, h, y, z, h), dict(dgate=x)),
                 ((x, z, h, None, z, None), dict(dw_after=w))):
        with pytest.raises(harp.HarpError):
            bwd(*a, **k)
    with pytest.raises(harp.HarpError):
        ops.norm_workspace(ctx, 4, 0)
    ctx.close()
