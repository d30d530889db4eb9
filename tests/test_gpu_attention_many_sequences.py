"""More sequences times kv heads than one launch has workgroups."""
import pytest

from attention_plan import plans


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
def test_a_million_sequences_of_one_token(harp, tmp_path, causal):
    """One key a query: its value is the result and its gradient the value's, to the bit; the score is the sum's logarithm; P (dP - D) is what
    two sums of 8 products in 32 bits differ by."""
    import torch
    from paper_2509_24859_amd import operators as ops
    batch, heads, head, t = 1 << 20, 24, 8, torch.bfloat16
    of_rows, of_keys = plans(str(tmp_path), [(batch, batch, batch, heads, heads, head, causal)])[0]
    assert of_keys["heads"] < heads and (of_rows["heads"] < heads or of_rows["paired"])       # two tiles a workgroup fit one launch
    ctx = harp.Context(0)
    q, k, v, do = (torch.randn(batch, heads, head, device="cuda").to(t) for _ in range(4))
    o, lse, dq, dk, dv = torch.empty_like(q), torch.empty(heads, batch, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    form = dict(batch=batch, causal=causal, scale=0.5, workspace=ops.attention_workspace(ctx, batch, batch, batch, heads, heads, head))
    ops.harp_attention_forward(ctx, q, k, v, o, lse=lse, **form)
    assert torch.equal(o, v)
    e = 2.0 ** -24
    score, terms = (0.5 * (q.double() * k).sum(2)).t(), (0.5 * (q.double() * k).abs().sum(2)).t()
    assert ((lse - score).abs() <= (65 * terms + 4 * score.abs() + 16) * e).all()
    ops.harp_attention_backward(ctx, q, k, v, o, lse, do, dq, dk, dv, **form)
    assert torch.equal(dv, do)
    room = 0.5 * 1.02 * 2 * 65 * e * (do.double() * v).abs().sum(2, keepdim=True)
    assert (dq.abs() <= room * k.abs()).all() and (dk.abs() <= room * q.abs()).all()
    ctx.close()
