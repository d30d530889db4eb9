"""Attention and its gradients over lengths that take the kernels through their steady loops: workgroups of 8 wavefronts with many tiles of
keys each, under the causal order the heads dealt out to the dies, and a heavy and a light tile in one workgroup.  Formulas in 64 bits, a
head at a time on the GPU; rooms as derived in test_gpu_attention.py.
"""
import math

import pytest

from attention_plan import plans

E = 2.0 ** -24
UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}

# lengths, heads, kv heads, head, causal, type; None for begins: sequences of equal length
CASES = [
    ((4090,), None, 32, 32, 128, True, "bfloat16"),
    ((4090,), None, 32, 32, 128, False, "float16"),
    ((2051, 2051), None, 24, 24, 64, True, "float16"),
    ((2309,), None, 48, 24, 96, True, "bfloat16"),
    ((3001, 3001), None, 64, 16, 128, True, "float16"),
    ((1500, 3, 2500, 0, 700), "packed", 16, 8, 128, True, "bfloat16"),
    ((2777, 1203), "packed", 12, 4, 96, False, "bfloat16"),
]


def _name(c):
    return "%s-%d.%dx%d%s-%s" % (".".join(map(str, c[0])), c[2], c[3], c[4], "-causal" if c[5] else "", c[6])


def test_the_cases_take_these_paths(tmp_path):
    """The steady loops of 8 wavefronts at each of the three widths, with sums that stay in one workgroup; two tiles in one, long ones, for
    even and odd numbers of places; heads dealt out to the dies, and shares."""
    calls = [(sum(n), sum(n), len(n), heads, kv, head, causal) for n, _, heads, kv, head, causal, _ in CASES]
    both = plans(str(tmp_path), calls)
    assert all(p["waves"] == 8 for pair in both for p in pair)
    assert {c[5] for c, (rows, _) in zip(calls, both) if rows["paired"] and rows["shares"] == 1 and c[4] % 8 == 0} == {64, 96, 128}
    assert {rows["tiles"] % 2 for rows, _ in both if rows["paired"]} == {0, 1}
    assert any(rows["shares"] == 1 and not c[6] and c[5] == 128 for c, (rows, _) in zip(calls, both))
    assert {keys["shares"] == 1 for c, (_, keys) in zip(calls, both) if c[6] and c[4] % 8 == 0} == {False, True}
    assert any(c[4] % 8 and not c[6] for c in calls)


def _of_head(q, k, v, do, causal, scale, u, rows):
    """What one head gives: o, lse, dq, dk, dv and by how much each may be off.  rows: queries that meet a kv head's keys."""
    import torch
    head, lq, lk = q.shape[1], q.shape[0], k.shape[0]
    seen = torch.ones(lq, lk, dtype=torch.bool, device=q.device)
    if causal:
        seen = seen.tril(lk - lq)
    t = lambda x: x.t().contiguous()  # noqa: E731
    s = scale * (q @ t(k))
    es = E * ((64 + head / 8) * scale * (q.abs() @ t(k.abs())) + 4 * s.abs())
    es = es.masked_fill(~seen, 0)
    s = s.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    worst = es.amax(1)
    o = p @ v
    o_room = (p @ v.abs()) * (u + 2 * worst + (64 + lk / 8) * E)[:, None]
    lse_room = worst + (16 + lk / 8) * E + 4 * E * lse.abs()
    dp, dp_mag = do @ t(v), do.abs() @ t(v.abs())
    delta, mag = (do * o).sum(1)[:, None], (do * o).abs().sum(1)[:, None]
    ds, w = p * (dp - delta), (64 + head / 8) * E
    rel = 2 * es + 16 * E + 4 * E * lse.abs()[:, None]
    off = p * (w * dp_mag + (u + w) * mag + rel * (dp.abs() + delta.abs())) + u * ds.abs()
    ds_mag = ds.abs() + off
    dq, dq_room = scale * ds @ k, scale * (off @ k.abs() + (64 + lk / 8) * E * ds_mag @ k.abs())
    dk, dk_room = scale * t(ds) @ q, scale * (t(off) @ q.abs() + (64 + rows / 8) * E * t(ds_mag) @ q.abs())
    dv, dv_room = t(p) @ do, t(p * (u + rel + (64 + rows / 8) * E)) @ do.abs()
    return (o, lse, dq, dk, dv), (o_room, lse_room, dq_room, dk_room, dv_room)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=_name)
def test_long(harp, case):
    import torch
    from paper_2509_24859_amd import operators as ops
    lengths, packed, heads, kv, head, causal, kind = case
    ctx, t, u, n = harp.Context(0), getattr(torch, kind), UNIT[kind], sum(lengths)
    gen = torch.Generator("cuda").manual_seed(n + head)
    draw = lambda h: torch.randn(n, h, head, device="cuda", generator=gen).to(t)  # noqa: E731
    q, do, k, v = draw(heads), draw(heads), draw(kv), draw(kv)
    at, group, scale = [sum(lengths[:i]) for i in range(len(lengths) + 1)], heads // kv, head ** -0.5
    form = dict(causal=causal, workspace=ops.attention_workspace(ctx, n, n, len(lengths), heads, kv, head))
    if packed:
        begin = torch.tensor(at, dtype=torch.int32, device="cuda")
        form |= dict(q_begin=begin, k_begin=begin)
    else:
        form |= dict(batch=len(lengths))
    f64 = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")  # noqa: E731
    shapes = ((n, heads, head), (heads, n), (n, heads, head), (n, kv, head), (n, kv, head))
    want, room = [f64(*s) for s in shapes], [f64(*s) for s in shapes]
    for b, length in enumerate(lengths):
        rows = slice(at[b], at[b + 1])
        if length == 0:
            continue
        for h in range(heads):
            x = [y[rows, i].double().contiguous() for y, i in ((q, h), (k, h // group), (v, h // group), (do, h))]
            for result, parts in ((want, 0), (room, 1)):
                values = _of_head(*x, causal, scale, u, length * group)[parts]
                result[0][rows, h], result[1][h, rows], result[2][rows, h] = values[:3]
                result[3][rows, h // group] += values[3]
                result[4][rows, h // group] += values[4]
    o, lse = torch.full_like(q, -7), torch.full((heads, n), -7.0, device="cuda")
    ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, **form)
    kept, kept_lse, grads = want[0].to(t), want[1].float(), [torch.full_like(x, -7) for x in (q, k, v)]
    ops.harp_attention_backward(ctx, q, k, v, kept, kept_lse, do, *grads, **form)
    for name, got, w, r in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads), want, room):
        if name != "lse":
            r = r + u * (w.abs() + r) + (2.0 ** -25 if kind == "float16" else 0)
        off = (got.double() - w).abs()
        print("%s: largest error over its room %.3f" % (name, (off / r).max().item()), flush=True)
        assert (off <= r).all(), (name, (off / r).max().item())
    again = [torch.full_like(x, -7) for x in (o, *grads)]          # the same bits again
    ops.harp_attention_forward(ctx, q, k, v, again[0], **form)
    ops.harp_attention_backward(ctx, q, k, v, kept, kept_lse, do, *again[1:], **form)
    assert all(torch.equal(x, y) for x, y in zip(again, (o, *grads)))
    ctx.close()
