"""Attention where one key outweighs the others: weights far below the largest count as much as the sum that they are divided by says.

All keys but a few have the same score, so that results are known without a matrix product.  Rooms are those of
test_gpu_attention.py: of the sum of p |v| half a unit of the type for the weights, twice what scores are off by and 64 + n / 8 roundings
to 32 bits; of the result half a unit, and in float16 half of its smallest step.
"""
import math

import pytest

E = 2.0 ** -24
UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def _run(harp, kind, head, tokens, heads, scores, values):
    """o and lse of `tokens` like queries, whose scores are `scores` exactly: 16 bits hold a quarter of them."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx, n, t = harp.Context(0), len(scores), getattr(torch, kind)
    q, k = torch.zeros(tokens, heads, head, dtype=t, device="cuda"), torch.zeros(n, heads, head, dtype=t, device="cuda")
    q[..., 0] = 4
    k[..., 0] = (scores / 4).to(t).cuda()[:, None]
    assert torch.equal(k[:, 0, 0].double().cpu() * 4, scores)
    v = values.to(t).cuda().expand(heads, n, head).transpose(0, 1)
    o, lse = torch.empty_like(q), torch.empty(heads, tokens, device="cuda")
    ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, scale=1.0, workspace=ops.attention_workspace(ctx, tokens, n, 1, heads, heads, head))
    p = torch.softmax(scores, 0)
    kept = v[:, 0].double().cpu()
    es = (64 + head / 8 + 4) * float(scores.abs().max()) * E
    sums = UNIT[kind] + 2 * es + (64 + n / 8) * E
    want, room = p @ kept, p @ kept.abs() * sums
    room = room + UNIT[kind] * (want.abs() + room) + (2.0 ** -25 if kind == "float16" else 0)
    off = (o.double().cpu() - want).abs()
    print("largest error over its room: %.3f" % (off / room).max().item(), flush=True)
    assert (off <= room).all(), (off / room).max()
    total = float(torch.logsumexp(scores, 0))
    assert (lse.double() - total).abs().max() <= es + (16 + n / 8) * E + 4 * E * abs(total)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("place", ["first", "middle", "last"])
@pytest.mark.parametrize("kind,head", [("float16", 64), ("float16", 96), ("float16", 128), ("bfloat16", 128)])
@pytest.mark.parametrize("above", [12.0, 15.0, 17.0])
def test_one_key_far_above_the_others(harp, above, kind, head, place):
    """e^-12, e^-15 and e^-17 are 2^-17.3, 2^-21.6 and 2^-24.5.  The key above has a value of 0, so that the result is the others'; all rows
    are full tiles, so that no share of the keys lacks it."""
    import torch
    n = 65537
    scores = torch.zeros(n, dtype=torch.float64)
    values = torch.rand(n, head, generator=torch.Generator().manual_seed(head)) + 0.5
    at = {"first": 0, "middle": n // 2, "last": n - 1}[place]
    scores[at], values[at] = above, 0
    _run(harp, kind, head, 4096, 16, scores, values)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,head", [("float16", 64), ("float16", 128), ("bfloat16", 96)])
@pytest.mark.parametrize("step", [0.5, 2.0, 2.0625, 2.125, 5.5, 5.75])
def test_scores_that_rise_a_little_at_a_time(harp, step, kind, head):
    """The reference that exponents are taken against may stay behind the largest score by some powers of two (2.08 nats are three, 5.55
    eight): weights reach the type's range then and do not leave it."""
    import torch
    n = 4096
    scores = torch.arange(8, dtype=torch.float64).repeat_interleave(n // 8) * step
    values = torch.randn(n, head, generator=torch.Generator().manual_seed(head)) * 100
    _run(harp, kind, head, 300, 4, scores, values)
