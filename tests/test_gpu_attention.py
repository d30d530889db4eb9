"""Attention and its gradients against their formulas in 64 bits.

Tolerances, with u half a unit of the type's last place (2^-8, 2^-11) and e = 2^-24.  A score is a sum of D products of 16-bit values
in 32 bits and two factors: off by es = ((64 + D / 8) times its sum of magnitudes + 4 times itself) e.  An exponential is then off by
es (relative) and 8 e more; weights are rounded to the type where they are multiplied.  So
  o       within sum of p |v| times (u + 2 max es + (64 + Lk / 8) e), and u of itself when it is stored
  lse     within max es + (16 + Lk / 8) e + 4 e of itself
  dP, D   sums of D products; D's come from o as it is stored: u of the sum of |dO o| more
  dS      P times what dP and D are off by, (2 es + 16 e) of P (|dP| + |D|), and u of itself when it is multiplied
  dQ, dK  sums over keys or queries of that times |k| or |q|, and (64 + n / 8) e of their own sum of magnitudes
  dV      sum of P |dO| times (u + 2 es + ...)
A result of float16 is at least 2^-25 off where it is small.  A gradient that is not added, a mask off by one or a wrong
factor is far outside: terms are of order one, these rooms a few thousandths of their sum.
"""
import math

import numpy as np
import pytest

from operator_context import HostContext, refused

E = 2.0 ** -24
UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def _case(q, k, heads=1, kv=1, head=64, causal=False, kind="bfloat16", counts=None, equal=False, layout="plain", scale=None):
    return dict(q=q, k=k, heads=heads, kv=kv, head=head, causal=causal, kind=kind, counts=counts, equal=equal, layout=layout, scale=scale)


CASES = [
    _case([1], [1]), _case([1], [1], head=8, kind="float16"), _case([1], [64], 4, 2), _case([5], [3], 2, 1, 40, kind="float16"),
    _case([32], [32], causal=True), _case([33], [65], 3, 3, 128), _case([64], [64], 2, 2, 128, True, "float16"),
    _case([100], [100], 8, 2, 96, True), _case([127], [130], 2, 1, 72, True), _case([129], [200], 6, 2, 80, kind="float16"),
    _case([256], [256], 2, 2, 128, True), _case([257], [300], 4, 4, 64, True, "float16"), _case([300], [129], 4, 1, 112, False),
    _case([70], [40], 2, 1, 64, True), _case([500], [100], 3, 1, 128, True),                     # rows that see no key
    _case([1], [5000], 8, 2, 128), _case([1] * 5, [700, 1, 64, 3000, 65], 16, 2, 64, kind="float16"), _case([7], [2500], 4, 4, 80, True),
    _case([3, 0, 40, 129, 1], [50, 7, 0, 200, 64], 6, 3, 64), _case([3, 20, 40, 129, 1], [50, 20, 41, 200, 64], 6, 3, 128, True, "float16"),
    _case([20, 30, 5], [64, 64, 64], 2, 1, 64, counts=[64, 0, 17]), _case([20, 70, 5], [90, 90, 90], 2, 2, 96, True, "float16", counts=[1, 77, 90]),
    _case([40] * 3, [70] * 3, 4, 2, 64, True, equal=True), _case([17] * 4, [33] * 4, 3, 3, 128, counts=[33, 1, 0, 20], equal=True),
    _case([90, 31], [100, 64], 4, 2, 64, True, layout="odd"), _case([90, 31], [100, 64], 4, 2, 128, layout="heads first"),
    _case([90, 31], [100, 64], 4, 2, 80, True, layout="fused"), _case([60], [70], 4, 2, 64, scale=3.0), _case([2] * 70, [3] * 70, 2, 1, 16, True),
    _case([1000], [77], 8, 8, 64), _case([40], [3000], 2, 2, 128, kind="float16"), _case([777, 500], [777, 500], 4, 1, 128, True),
]


def _id(c):
    return "%s-%s-%d.%dx%d%s%s%s" % (".".join(map(str, c["q"][:4])), ".".join(map(str, c["k"][:4])), c["heads"], c["kv"], c["head"],
                                     "-causal" if c["causal"] else "", "-" + c["layout"] if c["layout"] != "plain" else "",
                                     "-f16" if c["kind"] == "float16" else "")


def _begins(counts):
    return [0] + np.cumsum(counts).tolist()


class _Setup:
    """The case's tensors on the GPU, between two rows of no sequence each, and their values in 64 bits."""

    def __init__(self, harp, c, seed=0):
        import torch
        from paper_2509_24859_amd import operators as ops
        self.c, self.torch, self.ops, self.ctx = c, torch, ops, harp.Context(0)
        self.kind, self.rng = getattr(torch, c["kind"]), np.random.default_rng(seed + sum(c["q"]) * 31 + sum(c["k"]) + c["head"])
        self.lead = 0 if c["equal"] else 2
        self.q_at, self.k_at = ([self.lead + x for x in _begins(n)] for n in (c["q"], c["k"]))
        self.tq, self.tk = self.q_at[-1] + self.lead, self.k_at[-1] + self.lead
        self.used = c["counts"] or c["k"]
        h, kv, d = c["heads"], c["kv"], c["head"]
        draw = lambda *s: torch.from_numpy(self.rng.standard_normal(s)).to(self.kind).double().numpy()  # noqa: E731
        self.q, self.do, self.k, self.v = draw(self.tq, h, d), draw(self.tq, h, d), draw(self.tk, kv, d), draw(self.tk, kv, d)
        held = np.zeros(self.tk, dtype=bool)
        for b, n in enumerate(self.used):
            held[self.k_at[b]:self.k_at[b] + n] = True
        self.k[~held], self.v[~held] = math.nan, math.inf           # nothing may be taken from there
        self.scale = d ** -0.5 if c["scale"] is None else c["scale"]
        self.form = dict(causal=c["causal"], scale=c["scale"])
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        if c["equal"]:
            self.form["batch"] = len(c["q"])
        else:
            self.form |= dict(q_begin=i32(self.q_at), k_begin=i32(self.k_at))
        if c["counts"]:
            self.form["k_count"] = i32(c["counts"])
        self.form["workspace"] = ops.attention_workspace(self.ctx, self.tq, self.tk, len(c["q"]), h, kv, d)
        self.form["workspace"].fill_(0xFF)

    def put(self, values):
        """[tokens][heads][head] on the GPU; what is between holds -7."""
        torch, layout, (n, h, d) = self.torch, self.c["layout"], values.shape
        if layout == "heads first":
            view = torch.full((h, n, d), -7.0, dtype=self.kind, device="cuda").transpose(0, 1)
        elif layout == "odd":
            view = torch.full((1 + n * (h * (d + 3) + 1),), -7.0, dtype=self.kind, device="cuda")[1:].view(n, -1)[:, :h * (d + 3)].view(n, h, d + 3)[..., :d]
        elif layout == "fused":
            view = torch.full((n, 2 * h, d), -7.0, dtype=self.kind, device="cuda")[:, h:]
        else:
            view = torch.full((n, h, d), -7.0, dtype=self.kind, device="cuda")
        view.copy_(torch.from_numpy(values).to(self.kind))
        return view

    def sequences(self):
        """Per sequence and head: what the formulas give, and by how much a result may be off."""
        c, u = self.c, UNIT[self.c["kind"]]
        group = c["heads"] // c["kv"]
        for b, (lq, used) in enumerate(zip(c["q"], self.used)):
            rows, keys = slice(self.q_at[b], self.q_at[b] + lq), slice(self.k_at[b], self.k_at[b] + used)
            seen = np.ones((lq, used), dtype=bool)
            if c["causal"]:
                seen = np.arange(used)[None, :] <= np.arange(lq)[:, None] + used - lq
            for h in range(c["heads"]):
                q, k, v = self.q[rows, h], self.k[keys, h // group], self.v[keys, h // group]
                s = self.scale * (q @ k.T)
                es = E * ((64 + c["head"] / 8) * self.scale * (np.abs(q) @ np.abs(k).T) + 4 * np.abs(s))
                es = np.where(seen, es, 0)
                top = np.where(seen, s, -np.inf).max(1, initial=-np.inf)
                some = np.isfinite(top)
                p = np.where(seen, np.exp(s - np.where(some, top, 0)[:, None]), 0)
                total = p.sum(1)
                p = p / np.where(some, total, 1)[:, None]
                lse = np.where(some, top + np.log(np.where(some, total, 1)), -np.inf)
                worst = es.max(1, initial=0)
                o = p @ v
                o_room = (p @ np.abs(v)) * (u + 2 * worst + (64 + used / 8) * E)[:, None]
                lse_room = worst + (16 + used / 8) * E + 4 * E * np.where(some, np.abs(lse), 0)
                yield dict(b=b, h=h, kv=h // group, rows=rows, keys=keys, q=q, k=k, v=v, es=es, p=p, o=o, o_room=o_room, lse=lse, lse_room=lse_room)


def _within(got, want, room, kind, what):
    u = UNIT[kind]
    room = room + u * (np.abs(want) + room) + (2.0 ** -25 if kind == "float16" else 0)
    off = np.abs(got - want)
    assert np.isfinite(got).all() and (off <= room).all(), (what, np.unravel_index(np.argmax(off - room), off.shape), (off / np.maximum(room, 1e-300)).max())


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=_id)
def test_forward(harp, case):
    s = _Setup(harp, case)
    torch = s.torch
    o, lse = s.put(np.full(s.q.shape, -7.0)), torch.full((case["heads"], s.tq), -7.0, device="cuda")
    args = [s.put(x) for x in (s.q, s.k, s.v)]
    s.ops.harp_attention_forward(s.ctx, *args, o, lse=lse, **s.form)
    got, got_lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    for x in s.sequences():
        _within(got[x["rows"], x["h"]], x["o"], x["o_room"], case["kind"], ("o", x["b"], x["h"]))
        g = got_lse[x["h"], x["rows"]]
        none = np.isneginf(x["lse"])
        assert (np.isneginf(g) == none).all() and (np.abs(g[~none] - x["lse"][~none]) <= x["lse_room"][~none]).all(), ("lse", x["b"], x["h"])
        assert (got[x["rows"], x["h"]][none] == 0).all()
    if s.lead:                                                    # rows of no sequence
        for at in (slice(0, 2), slice(s.tq - 2, s.tq)):
            assert (got[at] == -7).all() and (got_lse[:, at] == -7).all()
    again = s.put(np.full(s.q.shape, -7.0))
    s.ops.harp_attention_forward(s.ctx, *args, again, **s.form)   # the same bits, without lse too
    assert torch.equal(o, again)
    s.ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1.0, 2.0 ** -12, 2.0 ** 9], ids=["", "small", "large"])
@pytest.mark.parametrize("case", CASES, ids=_id)
def test_gradients(harp, case, size):
    s = _Setup(harp, case, seed=1)
    torch, kind, u = s.torch, case["kind"], UNIT[case["kind"]]
    s.do = torch.from_numpy(s.do * size).to(s.kind).double().numpy()
    o, lse = np.zeros(s.q.shape), np.full((case["heads"], s.tq), 3.0)
    want = [np.zeros(s.q.shape), np.zeros(s.k.shape), np.zeros(s.k.shape)]
    room = [np.zeros(s.q.shape), np.zeros(s.k.shape), np.zeros(s.k.shape)]
    n = max(case["q"]) * case["heads"] // case["kv"]
    for x in s.sequences():
        rows, keys, h, kv, p, do = x["rows"], x["keys"], x["h"], x["kv"], x["p"], s.do[x["rows"], x["h"]]
        o[rows, h], lse[h, rows] = x["o"], x["lse"]
        dp, dp_mag = do @ x["v"].T, np.abs(do) @ np.abs(x["v"]).T
        delta, mag = (do * x["o"]).sum(1)[:, None], (np.abs(do) * np.abs(x["o"])).sum(1)[:, None]
        ds, w = p * (dp - delta), (64 + case["head"] / 8) * E
        rel = 2 * x["es"] + 16 * E + 4 * E * np.abs(np.where(np.isfinite(x["lse"]), x["lse"], 0))[:, None]
        off = p * (w * dp_mag + (u + w) * mag + rel * (np.abs(dp) + np.abs(delta))) + u * np.abs(ds)
        ds_mag = np.abs(ds) + off
        want[0][rows, h], room[0][rows, h] = s.scale * ds @ x["k"], s.scale * (off @ np.abs(x["k"]) + (64 + p.shape[1] / 8) * E * ds_mag @ np.abs(x["k"]))
        want[1][keys, kv] += s.scale * ds.T @ x["q"]
        room[1][keys, kv] += s.scale * (off.T @ np.abs(x["q"]) + (64 + n / 8) * E * ds_mag.T @ np.abs(x["q"]))
        want[2][keys, kv] += p.T @ do
        room[2][keys, kv] += (p * (u + rel + (64 + n / 8) * E)).T @ np.abs(do)
    args = [s.put(x) for x in (s.q, s.k, s.v, o)]
    lse, do = torch.from_numpy(lse).float().cuda(), s.put(s.do)
    out = [s.put(np.full(x.shape, -7.0)) for x in want]
    s.ops.harp_attention_backward(s.ctx, *args, lse, do, *out, **s.form)
    for name, g, w, r, at, counts in zip(("dq", "dk", "dv"), out, want, room, (s.q_at, s.k_at, s.k_at), (case["q"], case["k"], case["k"])):
        g = g.double().cpu().numpy()
        for b, m in enumerate(counts):
            rows = slice(at[b], at[b] + m)
            _within(g[rows], w[rows], r[rows], kind, (name, b))
        if s.lead:
            assert (g[:2] == -7).all() and (g[-2:] == -7).all()
    if case["counts"]:                                            # keys that are not used
        for b, m in enumerate(case["k"]):
            rest = slice(s.k_at[b] + s.used[b], s.k_at[b] + m)
            assert all((x[rest] == 0).all() for x in out[1:])
    if size == 1.0:                                               # the same bits again, and one gradient at a time
        for i in range(3):
            alone = [s.put(np.full(x.shape, -7.0)) if j == i else None for j, x in enumerate(want)]
            s.ops.harp_attention_backward(s.ctx, *args, lse, do, *alone, **s.form)
            assert torch.equal(alone[i], out[i])
    s.ctx.close()


@pytest.mark.gpu
def test_gradients_by_differences(harp):
    """The sum of o g along a direction of q, k and v, from the formula in 64 bits, against the gradients of both passes run one after
    the other.  The quotient's own error is below 1e-6 of the terms; each gradient is off by a few units of 2^-11 of its terms' sum."""
    c = _case([30], [45], 4, 2, 64, True, "float16")
    s = _Setup(harp, c, seed=2)
    torch = s.torch
    q, k, v, g = (s.put(x) for x in (s.q, s.k, s.v, s.do))
    o, lse = torch.empty_like(q), torch.empty(4, s.tq, device="cuda")
    s.ops.harp_attention_forward(s.ctx, q, k, v, o, lse=lse, **s.form)
    grads = [torch.empty_like(x) for x in (q, k, v)]
    s.ops.harp_attention_backward(s.ctx, q, k, v, o, lse, g, *grads, **s.form)
    at = {"q": slice(2, 32), "k": slice(2, 47), "v": slice(2, 47)}
    for name, grad in zip("qkv", grads):
        kept = getattr(s, name)
        way = s.rng.standard_normal(kept.shape)
        value = []
        for step in (1e-4, -1e-4):
            setattr(s, name, kept + step * way)
            value.append(sum((x["o"] * s.do[x["rows"], x["h"]]).sum() for x in s.sequences()))
        setattr(s, name, kept)
        terms = grad.double().cpu().numpy()[at[name]] * way[at[name]]
        assert abs(terms.sum() - (value[0] - value[1]) / 2e-4) <= (8 * 2.0 ** -11 + 1e-5) * np.abs(terms).sum(), name
    s.ctx.close()


@pytest.mark.gpu
def test_scores_far_apart(harp):
    """Scores of thousands, and a row whose first keys are far below its last: the reference that exponents are taken against moves."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    n, d = 300, 64
    q, k = torch.zeros(n, 1, d, device="cuda").half(), torch.zeros(n, 1, d, device="cuda").half()
    q[:, 0, 0] = 60
    k[:, 0, 0] = torch.linspace(-50, 50, n, device="cuda")
    v = torch.randn(n, 1, d, device="cuda").half()
    o, lse = torch.empty_like(q), torch.empty(1, n, device="cuda")
    ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, scale=1.0, workspace=ops.attention_workspace(ctx, n, n, 1, 1, 1, d))
    s = q[:, 0].double() @ k[:, 0].double().t().contiguous()
    want = torch.softmax(s, 1) @ v[:, 0].double()
    # scores are exact; exponents differ by up to 1e4, of which 32 bits keep 1e4 * 4 * 2^-24 after the factor
    assert ((o[:, 0].double() - want).abs() <= 2.0 ** -10 * want.abs() + (2.0 ** -11 + 3e-3) * (torch.softmax(s, 1) @ v[:, 0].double().abs())).all()
    assert ((lse[0].double() - torch.logsumexp(s, 1)).abs() <= 16 * 2.0 ** -24 * s.abs().max()).all()
    ctx.close()


@pytest.mark.gpu
def test_what_is_not_finite_stays_where_it_is_seen(harp):
    """A NaN in a query stays in its row, one in a key or value in the rows of its kv head; an infinite score makes its row NaN."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    q, k, v = (torch.randn(150, h, 64, device="cuda").bfloat16() for h in (4, 2, 2))
    ws = ops.attention_workspace(ctx, 150, 150, 1, 4, 2, 64)
    q[17, 1, 3] = math.nan
    v[149, 1, 5] = math.nan
    o, lse = torch.empty_like(q), torch.empty(4, 150, device="cuda")
    ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, workspace=ws)
    bad = torch.isnan(o)
    want = torch.zeros_like(bad)
    want[17, 1] = True
    want[:, 2:, 5] = True
    assert torch.equal(bad, want) and torch.isnan(lse).sum() == 1
    ctx.close()


@pytest.mark.gpu
def test_captured_with_lengths_that_change(harp):
    """A captured pass takes the begins and counts of each replay; two graphs share a workspace, one after the other."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    h, kv, d, tq, tk = 4, 2, 64, 200, 900
    q, do = (torch.randn(tq, h, d, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn(tk, kv, d, device="cuda").bfloat16() for _ in range(2))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    qb, kb, count = i32([0, 60, 130, 200]), i32([0, 300, 600, 900]), i32([300, 299, 1])
    form = dict(q_begin=qb, k_begin=kb, k_count=count, causal=True, workspace=ops.attention_workspace(ctx, tq, tk, 3, h, kv, d))
    new = lambda: ([torch.full_like(q, -7), torch.full((h, tq), -7.0, device="cuda")], [torch.full_like(x, -7) for x in (q, k, v)])  # noqa: E731

    def forward(out):
        ops.harp_attention_forward(ctx, q, k, v, out[0], lse=out[1], **form)

    def backward(out, grads):
        ops.harp_attention_backward(ctx, q, k, v, *out, do, *grads, **form)

    out, grads = new()
    forward(out)
    backward(out, grads)
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        forward(out)
    with torch.cuda.graph(second):
        backward(out, grads)
    for begins, counts in (([0, 60, 130, 200], [300, 299, 1]), ([0, 1, 1, 150], [2, 300, 300]), ([50, 199, 200, 200], [0, 0, 300])):
        qb.copy_(i32(begins))
        count.copy_(i32(counts))
        want, want_grads = new()
        forward(want)
        backward(want, want_grads)
        for t in (*out, *grads):
            t.fill_(-7)
        first.replay()
        second.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*want, *want_grads), (*out, *grads)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (*out, *grads):
        t.fill_(-7)
    torch.cuda.synchronize()
    ops.harp_attention_forward(ctx, q, k, v, *out, **form, stream=side)
    ops.harp_attention_backward(ctx, q, k, v, *out, do, *grads, **form, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*want, *want_grads), (*out, *grads)))
    ctx.close()


@pytest.mark.gpu
def test_begins_and_counts_out_of_range_touch_nothing_else(harp):
    """They are kept within the tokens by the kernels: what lies around the tensors stays as it is."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    h, kv, d, tq, tk = 2, 1, 64, 100, 120

    def inside(n, heads, fill):
        buf = torch.full((n + 200, heads, d), -7.0, device="cuda").bfloat16()
        buf[100:-100] = fill
        return buf, buf[100:-100]

    ws = ops.attention_workspace(ctx, tq, tk, 3, h, kv, d)
    for qb, kb, count in (([-5, 1000, 50, 70], [0, 40, 500, 1 << 30], [-1, 1 << 30, 7]), ([90, 10, 100, 100], [120, 0, -(1 << 31), 60], [5, 5, 5]),
                          ([(1 << 31) - 1] * 4, [-(1 << 31)] * 4, [1, 2, 3])):
        q, k, v, do = (inside(n, x, 1.0)[1] for n, x in ((tq, h), (tk, kv), (tk, kv), (tq, h)))
        bufs = [inside(n, x, -7.0) for n, x in ((tq, h), (tq, h), (tk, kv), (tk, kv))]
        form = dict(workspace=ws) | {n: torch.tensor(x, dtype=torch.int32, device="cuda") for n, x in (("q_begin", qb), ("k_begin", kb), ("k_count", count))}
        lse = torch.zeros(h, tq, device="cuda")
        ops.harp_attention_forward(ctx, q, k, v, bufs[0][1], lse=lse, **form)
        ops.harp_attention_backward(ctx, q, k, v, bufs[0][1], lse, do, *(b[1] for b in bufs[1:]), **form)
        torch.cuda.synchronize()
        assert all((b[0][:100] == -7).all() and (b[0][-100:] == -7).all() for b in bufs)
    ctx.close()


def _plain(q, k, v, group, causal=False):
    """o of one sequence in 64 bits, and the sum of p |v|."""
    import torch
    q, k, v = (x.double() for x in (q, k, v))
    out, mag = torch.empty_like(q), torch.empty_like(q)
    for h in range(q.shape[1]):
        s = q[:, h].contiguous() @ k[:, h // group].t().contiguous() * q.shape[2] ** -0.5
        if causal:
            s = s.masked_fill(torch.ones_like(s).triu(1 + s.shape[1] - s.shape[0]).bool(), -math.inf)
        p = torch.softmax(s, 1)
        out[:, h], mag[:, h] = p @ v[:, h // group].contiguous(), p @ v[:, h // group].abs().contiguous()
    return out, mag


def _near(got, want, mag):
    """Weights and result rounded to 2^-8, scores' and sums' roundings within 2^-10 of the terms at these sizes."""
    assert ((got.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -10) * mag + 2.0 ** -8 * want.abs()).all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits(harp):
    """Keys and values 65,536 elements apart: the last ones begin behind 2^31 elements.  Queries and their gradients likewise."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    n, far = 34000, 65536
    buf = torch.empty(n, far, dtype=torch.bfloat16, device="cuda")
    heads = lambda at, rows: buf[:rows, at:at + 128].unflatten(1, (2, 64))  # noqa: E731
    k, v, dk, dv = (heads(at, n) for at in (0, 1000, 2000, 3000))
    k.copy_(torch.randn(n, 2, 64, device="cuda"))
    v.copy_(torch.randn(n, 2, 64, device="cuda"))
    q, do = (torch.randn(3, 4, 64, device="cuda").bfloat16() for _ in range(2))
    o, dq, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(4, 3, device="cuda")
    ws = ops.attention_workspace(ctx, 3, n, 1, 4, 2, 64)
    ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, workspace=ws)
    _near(o, *_plain(q, k, v, 2))
    ops.harp_attention_backward(ctx, q, k, v, o, lse, do, dq, dk, dv, workspace=ws)
    near = [torch.empty_like(x, memory_format=torch.contiguous_format) for x in (k, v)]
    dq2 = torch.empty_like(dq)
    ops.harp_attention_backward(ctx, q, k.contiguous(), v.contiguous(), o, lse, do, dq2, *near, workspace=ws)
    assert torch.equal(dq, dq2) and torch.equal(dk, near[0]) and torch.equal(dv, near[1])
    many = heads(4000, n)                                        # as queries, of a few keys
    many.copy_(torch.randn(n, 2, 64, device="cuda"))
    out, lse = heads(5000, n), torch.empty(2, n, device="cuda")
    ops.harp_attention_forward(ctx, many, k[:5], v[:5], out, lse=lse, workspace=ops.attention_workspace(ctx, n, 5, 1, 2, 2, 64))
    _near(out, *_plain(many, k[:5], v[:5], 1))
    ctx.close()


@pytest.mark.gpu
def test_begins_on_one_side_and_keys_that_heads_share(harp):
    """Queries packed, keys of equal lengths; one head's keys seen as four by a distance of 0."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    q, k, v = (torch.randn(n, h, 64, device="cuda").bfloat16() for n, h in ((100, 4), (90, 1), (90, 1)))
    at = [0, 17, 17, 100]
    begin = torch.tensor(at, dtype=torch.int32, device="cuda")
    for kv in (1, 4):
        o = torch.empty_like(q)
        wide = [x.expand(90, kv, 64) for x in (k, v)]
        ops.harp_attention_forward(ctx, q, *wide, o, q_begin=begin, workspace=ops.attention_workspace(ctx, 100, 90, 3, 4, kv, 64))
        for b in range(3):
            rows, keys = slice(at[b], at[b + 1]), slice(30 * b, 30 * b + 30)
            _near(o[rows], *_plain(q[rows], k[keys], v[keys], 4))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [65, 1500, 3000])
def test_many_sequences(harp, batch):
    """More than a wavefront's lanes, and more than one turn of them; some empty, one long."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    rng = np.random.default_rng(batch)
    lengths = rng.integers(0, 9, batch)
    lengths[batch // 2] = 700
    at = [0] + np.cumsum(lengths).tolist()
    n = at[-1]
    q, k, v, do = (torch.randn(n, h, 64, device="cuda").bfloat16() for h in (2, 1, 1, 2))
    begin = torch.tensor(at, dtype=torch.int32, device="cuda")
    form = dict(q_begin=begin, k_begin=begin, causal=True, workspace=ops.attention_workspace(ctx, n, n, batch, 2, 1, 64))
    o, lse = torch.full_like(q, 7), torch.empty(2, n, device="cuda")
    grads = [torch.full_like(x, 7) for x in (q, k, v)]
    ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, **form)
    ops.harp_attention_backward(ctx, q, k, v, o, lse, do, *grads, **form)
    for b in (0, 1, 31, 63, 64, batch // 2 - 1, batch // 2, batch // 2 + 1, batch - 2, batch - 1):
        rows = slice(at[b], at[b + 1])
        if at[b] == at[b + 1]:
            continue
        _near(o[rows], *_plain(q[rows], k[rows], v[rows], 2, True))
        m = at[b + 1] - at[b]
        alone = [torch.empty_like(x[rows]) for x in (q, k, v)]
        ops.harp_attention_backward(ctx, q[rows], k[rows], v[rows], o[rows], lse[:, rows].contiguous(), do[rows], *alone, causal=True,
                                    workspace=ops.attention_workspace(ctx, m, m, 1, 2, 1, 64))
        # sums may be shared out otherwise: the same to their roundings, half a unit of each and 2^-10 of the largest
        assert all(((x[rows].double() - y.double()).abs() <= 2.0 ** -8 * (x[rows].double().abs() + y.double().abs()) / 2 + 2.0 ** -10 * y.abs().max()).all()
                   for x, y in zip(grads, alone))
    ctx.close()


@pytest.mark.gpu
def test_no_tokens(harp):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    b16 = dict(dtype=torch.bfloat16, device="cuda")
    q, k, none_q, none_k = torch.randn(5, 2, 64, **b16), torch.randn(7, 1, 64, **b16), torch.empty(0, 2, 64, **b16), torch.empty(0, 1, 64, **b16)
    o, lse, dq, dk, dv = torch.empty_like(q), torch.empty(2, 5, device="cuda"), torch.ones_like(q), torch.ones_like(k), torch.ones_like(k)
    ws = lambda a, b: ops.attention_workspace(ctx, a, b, 1, 2, 1, 64)  # noqa: E731
    ops.harp_attention_forward(ctx, none_q, k, k, none_q, workspace=ws(0, 7))
    ops.harp_attention_backward(ctx, none_q, k, k, none_q, lse[:, :0].contiguous(), none_q, none_q, dk, dv, workspace=ws(0, 7))
    assert (dk == 0).all() and (dv == 0).all()
    ops.harp_attention_forward(ctx, q, none_k, none_k, o, lse=lse, workspace=ws(5, 0))
    assert (o == 0).all() and torch.isneginf(lse).all()
    ops.harp_attention_backward(ctx, q, none_k, none_k, o, lse, q, dq, none_k, none_k, workspace=ws(5, 0))
    assert (dq == 0).all()
    ctx.close()


def test_refusals(monkeypatch):
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = HostContext()
    b = torch.bfloat16
    q, k, o = torch.zeros(6, 4, 16, dtype=b), torch.zeros(9, 2, 16, dtype=b), torch.zeros(6, 4, 16, dtype=b)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    lse = torch.zeros(4, 6)
    ws = ops.attention_workspace(ctx, 6, 9, 1, 4, 2, 16)
    ws = ws[-ws.data_ptr() % 256:] if ws.data_ptr() % 256 else ws
    big = torch.zeros(1 << 16, dtype=torch.uint8)
    big = big[-big.data_ptr() % 256:]
    fwd = lambda *a, **kw: refused(monkeypatch, ops.harp_attention_forward, ctx, *a, **(dict(workspace=big) | kw))  # noqa: E731
    for a, kw in (((q.float(), k.float(), k.float(), o.float()), {}), ((q, k.half(), k, o), {}), ((q, k, k[:8], o), {}), ((q, k, k, o[:5]), {}),
                  ((q[..., :12], k[..., :12], k[..., :12], o[..., :12]), {}), ((q[:, :3], k, k, o[:, :3]), {}), ((q[0], k, k, o), {}),
                  ((q, k, k, o), dict(lse=torch.zeros(4, 5))), ((q, k, k, o), dict(lse=lse.double())), ((q, k, k, o), dict(scale=0.0)),
                  ((q, k, k, o), dict(scale=-1.0)), ((q, k, k, o), dict(scale=math.nan)), ((q, k, k, o), dict(batch=2)), ((q, k, k, o), dict(batch=0)),
                  ((q, k, k, o), dict(q_begin=i32(0, 3, 6), k_begin=i32(0, 9))), ((q, k, k, o), dict(q_begin=i32(0, 3, 6), batch=3)),
                  ((q, k, k, o), dict(q_begin=i32(0, 6).long())), ((q, k, k, o), dict(k_count=i32(1, 2))), ((q, k, k, o), dict(workspace=None)),
                  ((q, k, k, o), dict(workspace=big[1:])), ((q, k, k, o), dict(workspace=big[:256])),
                  ((q, k, k, o[:1].expand(6, 4, 16)), {}), ((q, k, k, torch.zeros(16, 4, 6, dtype=b).permute(2, 1, 0)), {})):
        fwd(*a, **kw)
    wide = torch.zeros(2, 2, 136, dtype=b)
    fwd(wide, wide, wide, wide)
    bwd = lambda *a, **kw: refused(monkeypatch, ops.harp_attention_backward, ctx, *a, **(dict(workspace=big) | kw))  # noqa: E731
    for a, kw in (((q, k, k, o, None, o, q, k, k), {}), ((q, k, k, o, lse, None, q, k, k), {}), ((q, k, k, o, lse, o, k, k, k), {}),
                  ((q, k, k, o, lse, o, q, q, k), {}), ((q, k, k, None, lse, o, q, k, k), {}), ((q, k, k, o, lse, o, q, k[:1].expand(9, 2, 16), k), {})):
        bwd(*a, **kw)
    for sizes in ((-1, 9, 1, 4, 2, 16), (1 << 30, 9, 1, 4, 2, 16), (6, 9, 0, 4, 2, 16), (6, 9, 1, 4, 3, 16), (6, 9, 1, 4, 2, 12), (6, 9, 1, 4, 2, 136),
                  (6, 9, 1, 0, 1, 16), (1 << 29, 9, 1, 4, 2, 16)):
        refused(monkeypatch, ops.attention_workspace, ctx, *sizes)


def test_results_over_operands_are_refused(monkeypatch):
    import torch
    from paper_2509_24859_amd import binding, operators as ops
    ctx, b = HostContext(), torch.bfloat16
    new = lambda n, h: torch.zeros(n, h, 16, dtype=b)  # noqa: E731
    q, k, v, o, do, dq, dk, dv, lse = new(6, 4), new(9, 2), new(9, 2), new(6, 4), new(6, 4), new(6, 4), new(9, 2), new(9, 2), torch.zeros(4, 6)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:]
    assert refused(monkeypatch, ops.harp_attention_forward, ctx, q, k, v, q, workspace=ws) == binding.ERR_INVALID_ARG
    for out in ((q, dk, dv), (do, dk, dv), (o, dk, dv), (dq, k, dv), (dq, dk, v), (dq, dk, dk)):
        assert refused(monkeypatch, ops.harp_attention_backward, ctx, q, k, v, o, lse, do, *out, workspace=ws) == binding.ERR_INVALID_ARG
    # times log2(e) it is beyond 32 bits
    assert refused(monkeypatch, ops.harp_attention_forward, ctx, q, k, v, o, scale=3e38, workspace=ws) == binding.ERR_INVALID_ARG


@pytest.mark.gpu
def test_begins_that_do_not_rise_stay_within_the_tensors(harp):
    """1,024 sequences of which every other one claims all 2^29 rows, 2^22 tiles of 128 each: together more than 31 bits hold.  No keys are
    anybody's, so queries' gradients are not asked for and keys' stay as they were."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx, b, tokens, heads, n = harp.Context(0), torch.bfloat16, 1 << 25, 16, 1024
    one = torch.ones(1, 1, 8, dtype=b, device="cuda")
    q = one.expand(tokens, heads, 8)
    k = torch.ones(n, 2, 8, dtype=b, device="cuda")
    lse = torch.zeros(heads, tokens, device="cuda")
    dk, dv = torch.full_like(k, -7), torch.full_like(k, -7)
    q_begin = torch.tensor([0, tokens] * (n // 2) + [0], dtype=torch.int32, device="cuda")
    need = ops.attention_workspace(ctx, tokens, n, n, heads, 2, 8).numel()
    lent = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    ops.harp_attention_backward(ctx, q, k, k, q, lse, q, None, dk, dv, q_begin=q_begin, k_begin=torch.zeros(n + 1, dtype=torch.int32, device="cuda"),
                                workspace=lent[:need])
    torch.cuda.synchronize()
    assert (dk == -7).all() and (dv == -7).all() and (lent[need:] == 0x5A).all()
    # lse 0 and dO = O of ones: 8 a row, whatever came of the other sequences
    delta = lent[:tokens * heads * 4].view(torch.float32)
    assert (delta == 8).all()


@pytest.mark.gpu
@pytest.mark.parametrize("head", [64, 96, 128])
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
def test_queries_without_keys_have_no_part_in_gradients(harp, kind, head):
    """70 and 600 queries, causal, of 40 and 300 keys: whatever the first 30 and 300 and their gradients hold, the others' results and the
    keys' are the same bits.  Gradients of a few hundred, so that float16 has to scale them.  A key that only the last query sees, and
    is not finite, leaves the queries without keys their zeros."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx, t = harp.Context(0), getattr(torch, kind)
    rng = np.random.default_rng(head)
    draw = lambda n, h: torch.from_numpy(rng.standard_normal((n, h, head))).to(t).cuda()  # noqa: E731
    q, do, k, v = draw(670, 4), draw(670, 4) * 256, draw(340, 2), draw(340, 2)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    form = dict(q_begin=i32(0, 70, 670), k_begin=i32(0, 40, 340), causal=True, workspace=ops.attention_workspace(ctx, 670, 340, 2, 4, 2, head))
    empty = torch.zeros(670, dtype=torch.bool, device="cuda")
    empty[:30] = empty[70:370] = True
    results = []
    for fill in (0.0, math.nan, math.inf, 6e4):
        q[empty], do[empty] = fill, fill
        o, lse, grads = torch.empty_like(q), torch.empty(4, 670, device="cuda"), [torch.empty_like(x) for x in (q, k, v)]
        ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, **form)
        ops.harp_attention_backward(ctx, q, k, v, o, lse, do, *grads, **form)
        assert (o[empty] == 0).all() and (lse[:, empty] == -math.inf).all() and (grads[0][empty] == 0).all(), fill
        assert all(torch.isfinite(x).all() for x in grads), fill
        results.append([o, lse] + grads)
        assert all(torch.equal(x, y) for x, y in zip(results[0], results[-1])), fill
    k[39], v[339] = math.nan, math.inf
    o, lse, dq = torch.empty_like(q), torch.empty(4, 670, device="cuda"), torch.empty_like(q)
    ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, **form)
    ops.harp_attention_backward(ctx, q, k, v, o, lse, do, dq, None, None, **form)
    assert (o[empty] == 0).all() and (lse[:, empty] == -math.inf).all() and (dq[empty] == 0).all()
    ctx.close()


@pytest.mark.gpu
def test_what_is_not_finite_in_one_sequence_leaves_the_others_as_they_are(harp):
    """float16, gradients of a few hundred: a gradient or value of one sequence that is not finite changes no bit of the other's."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx, t = harp.Context(0), torch.float16
    q, do, k, v = (torch.randn(200, 2, 64, device="cuda").to(t) for _ in range(4))
    do *= 256
    form = dict(batch=2, workspace=ops.attention_workspace(ctx, 200, 200, 2, 2, 2, 64))
    results = []
    for bad in (0.0, math.nan, math.inf):
        do[3, 1, 5], v[40, 0, 7] = bad, 0.0
        for of_v in (0.0, bad):
            v[40, 0, 7] = of_v
            o, lse, grads = torch.empty_like(q), torch.empty(2, 200, device="cuda"), [torch.empty_like(x) for x in (q, k, v)]
            ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, **form)
            ops.harp_attention_backward(ctx, q, k, v, o, lse, do, *grads, **form)
            results.append([x[100:] for x in [o] + grads])
            assert all(torch.isfinite(x).all() for x in results[-1]), bad
            assert all(torch.equal(x, y) for x, y in zip(results[0], results[-1])), bad
    ctx.close()
