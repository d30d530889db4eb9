"""The norms' gradients where a workgroup works on several rows at a time: rows of few channels, gates' groups of one to
all rows, a last group cut short, workgroups whose last turn is not full; with and without biases, which are different
kernels.  The formula in 64 bits and the tolerances are those of the norms' other tests: a sum over rows adds one rounding
a row, in whatever order they are added.
"""
import numpy as np
import pytest

from test_gpu_norm import EPS, UNIT, _backward, _case, _on_gpu, _values, _within

pytestmark = pytest.mark.gpu

CASES = [
    # groups put together, more of them than teams, the last turn or group not full
    _case(7000, 40, "bfloat16", "layer", "rms", per=1, gate_act="sigmoid"), _case(5000, 72, "float16", "rms", "layer", per=3),
    _case(3000, 300, "float32", "layer", "layer", per=2, gate_act="sigmoid"), _case(2000, 1155, "float32", "layer", "layer", per=2),
    _case(1500, 520, "bfloat16", "rms", "rms", per=1), _case(1037, 1600, "float16", "layer", "none", per=3),
    _case(700, 3080, "bfloat16", "rms", "layer", per=2, gate_act="sigmoid"), _case(300, 6200, "bfloat16", "rms", "rms", per=1),
    # groups split, slabs of the last one empty; a slab a group
    _case(1999, 200, "bfloat16", "rms", "rms", per=700, gate_act="sigmoid"), _case(13001, 24, "float32", "rms", "layer", per=50),
    _case(2313, 450, "float16", "layer", "layer", per=257), _case(1100, 1024, "bfloat16", "none", "rms", per=999),
    # no gate; fewer rows than teams
    _case(6001, 128, "bfloat16", "layer", "rms"), _case(4000, 257, "float32"), _case(11, 64, "float16", "rms", "layer"),
    _case(13, 33, "bfloat16", "layer", "layer", per=5), _case(1, 100, "float32", "rms", "rms", per=1),
]


@pytest.mark.parametrize("biases", (True, False), ids=("biases", "weights"))
@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(str(x) for x in list(c.values())[:6]))
def test_rows_at_a_time(harp, c, biases):
    import torch
    from paper_2509_24859_amd import operators as ops
    if not biases:
        c = dict(c, without=("b_after", "b_before"))
    ctx = harp.Context(0)
    v = _values(c, np.random.default_rng(3))
    kind = getattr(torch, c["type"])
    vec = {n: _on_gpu(v[n], torch.float32) for n in ("scale", "w_after", "b_after", "w_before", "b_before")}
    t = {n: _on_gpu(v[n], kind) for n in ("dh", "dz", "h", "y", "gate")}
    if c["before"] == "none":
        v["dz"] = t["dz"] = None

    def run():
        names = ("dw_after", "dscale", "dw_before") + (("db_after", "db_before") if biases else ())
        out = {n: torch.full((c["cols"],), -7.0, device="cuda") for n in names}
        if c["per"]:
            out["dgate"] = torch.full(v["gate"].shape, -7.0, dtype=kind, device="cuda")
        dx, dy = (torch.full((c["rows"], c["cols"]), -7.0, dtype=kind, device="cuda") for _ in range(2))
        workspace = ops.norm_workspace(ctx, c["rows"], c["cols"], c["per"])
        workspace.view(torch.uint8).fill_(0xff)          # NaN: what is not written is not read
        ops.harp_norm_backward(ctx, t["dh"], t["dz"], t["h"], t["y"], dx, dy, after=c["after"], before=c["before"], gate=t["gate"],
                               rows_per_gate=c["per"] or 1, gate_act=c["gate_act"], eps=EPS, workspace=workspace, **vec, **out)
        return dict(out, dx=dx, dy=dy)

    got, again = run(), run()
    want = _backward(c, v)
    for name, value in got.items():
        assert torch.equal(value, again[name]), name
        value = value.double().cpu().numpy()
        if name not in want:
            assert name in ("dw_before", "db_before") and (value == 0).all(), name
            continue
        whole = name in ("dx", "dy", "dgate")
        _within(value, *want[name], 300 + (0 if name in ("dx", "dy") else c["rows"]), UNIT[c["type"]] if whole else 0.0, name)
    ctx.close()


@pytest.mark.parametrize("rows", (1, 2, 13, 300))
def test_a_gate_for_more_rows_than_there_are(harp, rows):
    """One gate for everything, however many rows it would be for: the same bits as for as many as there are."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    gate = torch.randn(1, 72, device="cuda")
    dh, dz, h, y = (torch.randn(rows, 72, device="cuda") for _ in range(4))
    got = []
    for per in (rows, rows + 1, 2 ** 62, 2 ** 63 - 1):
        out = [torch.full((rows, 72), -7.0, device="cuda") for _ in range(3)]
        dgate, dscale = torch.full((1, 72), -7.0, device="cuda"), torch.full((72,), -7.0, device="cuda")
        ops.harp_norm_forward(ctx, h, y, out[0], torch.empty_like(h), gate=gate, rows_per_gate=per)
        ops.harp_norm_backward(ctx, dh, dz, h, y, out[1], out[2], gate=gate, rows_per_gate=per, dgate=dgate, dscale=dscale,
                               workspace=ops.norm_workspace(ctx, rows, 72, per))
        got.append(out + [dgate, dscale])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
    ctx.close()
