"""The example that runs a decoder layer's operators together: its gradients, a captured step, its rows in a plan."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _norms(v, h, y):
    norm = lambda x, w: x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * w  # noqa: E731
    h = h + v["scale"] * norm(y, v["w_after"])
    return h, norm(h, v["w_before"])


def _attention(op, v, h, a):
    """The operator in 64 bits, with torch's differentiation."""
    import torch
    qkv = (a @ v["qkv"].t()).view(op.n, -1, op.d)
    each = op.n // op.sequences
    angle = (torch.arange(op.n) % each).double()[:, None] * op.frequencies.cpu()[None, :]
    c, s = torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]
    x, y = qkv[:, :op.heads + op.kv, :op.d // 2], qkv[:, :op.heads + op.kv, op.d // 2:]
    turned = torch.cat((x * c - y * s, y * c + x * s), 2)
    out = []
    for b in range(op.sequences):
        rows, heads = slice(b * each, (b + 1) * each), []
        for i in range(op.heads):
            k = op.heads + i // (op.heads // op.kv)
            score = turned[rows, i] @ turned[rows, k].t() * op.d ** -0.5
            score = score.masked_fill(torch.ones(each, each).triu(1).bool(), -float("inf"))
            heads.append(torch.softmax(score, 1) @ qkv[rows, k + op.kv])
        out.append(torch.cat(heads, 1))
    return _norms(v, h, torch.cat(out) @ v["out"].t())


def _mlp(op, v, h, a):
    z = a @ v["up"].t()
    f = z.shape[1] // 2
    return _norms(v, h, (z[:, :f].sigmoid() * z[:, :f] * z[:, f:]) @ v["down"].t())


@pytest.fixture
def made(harp):
    import torch
    import decoder_layer
    ctx = harp.Context(0)
    torch.manual_seed(3)
    yield ctx, {"attention": decoder_layer.Attention(ctx, 256, 192, 8, 2, sequences=2), "mlp": decoder_layer.GatedMlp(ctx, 256, 192, 328)}
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["attention", "mlp"])
def test_gradients_of_the_whole_operator(made, name):
    """Up to eight tensors of 16 bits lie between the operators of a chain, and weights of an attention are rounded on their way: each is
    off by half a unit, 2^-8 of its values at most, so the results are within 9 x 2^-8 of their norm."""
    import torch
    ctx, ops = made
    op, want_of = ops[name], _attention if name == "attention" else _mlp
    h, a, dh, da = (torch.randn(op.n, op.c, device="cuda").bfloat16() for _ in range(4))
    for k in range(2):                                    # two micro-batches: sums of two
        got_h, got_a = (t.clone() for t in op.forward(h, a))
        dx, dz = op.backward(a, dh, da, first=k == 0)
    v = {k: (op.low[k] if k in op.low else p).double().cpu().requires_grad_() for k, p in op.master.items()}
    H, A = (t.double().cpu().requires_grad_() for t in (h, a))
    want_h, want_a = want_of(op, v, H, A)
    ((want_h * dh.double().cpu()).sum() + (want_a * da.double().cpu()).sum()).backward()
    pairs = [("h", got_h, want_h, 1), ("a", got_a, want_a, 1), ("dh", dx, H.grad, 1), ("da", dz, A.grad, 1)]
    pairs += [("d" + k, op.grad[k], v[k].grad, 2) for k in op.master]
    for what, got, want, times in pairs:
        off = (got.double().cpu() - times * want).norm() / (times * want).norm()
        assert off < 9 * 2.0 ** -8, (what, off.item())


@pytest.mark.gpu
def test_a_layer_captured_and_replayed(made):
    """Both operators forward and back in one graph, with eager steps of the same buffers before, between and after its replays."""
    import torch
    ctx, ops = made
    first, second = ops["attention"], ops["mlp"]
    h, a, dh, da = (torch.randn(first.n, first.c, device="cuda").bfloat16() for _ in range(4))

    def layer():
        h1, a1 = first.forward(h, a)
        out = second.forward(h1, a1)
        dh1, da1 = second.backward(a1, dh, da, first=True)
        return (*out, *first.backward(a, dh1, da1, first=True), *first.grad.values(), *second.grad.values())

    out = layer()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for _ in range(3):
        for t in (h, a, dh, da):
            t.copy_(torch.randn_like(t))
        want = [t.clone() for t in layer()]
        for t in out:
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, out))
        first.step(1e-3)
        second.step(1e-3)


@pytest.mark.gpu
def test_measured_rows_are_planned(made):
    import decoder_layer
    import mlp_stage
    ctx, ops = made
    rows = [(100.2, 200.0, ops["attention"].bytes()), (150.0, 300.0, ops["mlp"].bytes())]
    p = decoder_layer.problem(rows, 3)
    assert p.fwd_us.tolist() == [[101, 150] * 3] and p.bwd_us.tolist() == [[200, 300] * 3]
    assert p.param_bytes.tolist() == [rows[0][2][0], rows[1][2][0]] * 3 and p.stash_bytes.tolist() == [rows[0][2][1], rows[1][2][1]] * 3
    best = mlp_stage.plan(ctx, decoder_layer.problem(rows, 20))
    assert best is not None and best["cuts"][-1] == 40
