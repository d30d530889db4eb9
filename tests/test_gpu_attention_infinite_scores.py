"""Queries whose scores are all -infinity, and those that are -infinity themselves."""
import math

import pytest


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("kind,head,key", [("bfloat16", 64, -math.inf), ("float16", 128, -math.inf), ("bfloat16", 96, -1e30)])
def test_keys_that_make_every_score_minus_infinity(harp, kind, head, key, causal):
    """The first sequence's keys are -infinity, or 32 bits do not hold their product, in a channel where its queries are positive: no result and
    no gradient of queries, none of keys and values that are finite either, and the second's results are the bits that it has alone."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx, t = harp.Context(0), getattr(torch, kind)
    gen = torch.Generator("cuda").manual_seed(head)
    q, do, k, v = (torch.randn(400, h, head, device="cuda", generator=gen).to(t) for h in (4, 4, 2, 2))
    q[:200, :, 0] = q[:200, :, 0].abs() + 1 if math.isinf(key) else 1e30
    k[:200, :, 0] = key
    results = []
    for b, rows in ((2, slice(0, 400)), (1, slice(200, 400))):
        of = [x[rows] for x in (q, k, v)]
        form = dict(batch=b, causal=causal, workspace=ops.attention_workspace(ctx, 200 * b, 200 * b, b, 4, 2, head))
        o, lse, grads = torch.full_like(of[0], 7), torch.full((4, 200 * b), 7.0, device="cuda"), [torch.full_like(x, 7) for x in of]
        ops.harp_attention_forward(ctx, *of, o, lse=lse, **form)
        ops.harp_attention_backward(ctx, *of, o, lse, do[rows], *grads, **form)
        results.append([o, lse.t(), *grads])
    both, alone = results
    assert (both[1][:200] == -math.inf).all() and (both[0][:200] == 0).all() and (both[2][:200] == 0).all()
    if math.isfinite(key):
        assert (both[3][:200] == 0).all() and (both[4][:200] == 0).all()
    assert all(torch.isfinite(x[200:]).all() for x in both)
    assert torch.equal(both[0][200:], alone[0]) and torch.equal(both[1][200:], alone[1])
    ctx.close()


@pytest.mark.gpu
def test_a_query_that_is_not_finite_stays_in_its_row(harp):
    """Forward; whatever its scores are."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    q, k, v = (torch.randn(150, 2, 64, device="cuda").bfloat16() for _ in range(3))
    k[:, :, 0] = k[:, :, 0].abs() + 1
    ws, results = ops.attention_workspace(ctx, 150, 150, 1, 2, 2, 64), []
    for x in (0.0, -math.inf):
        q[33, 1, 0] = x
        o, lse = torch.empty_like(q), torch.empty(2, 150, device="cuda")
        ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, causal=True, workspace=ws)
        results.append((o, lse))
    assert (results[1][0][33, 1] == 0).all() and results[1][1][1, 33] == -math.inf
    results[1][0][33, 1], results[1][1][1, 33] = results[0][0][33, 1], results[0][1][1, 33]
    assert all(torch.equal(x, y) for x, y in zip(*results))
    ctx.close()
