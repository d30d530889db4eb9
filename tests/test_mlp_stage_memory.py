"""What a device lends to the operators of its stage is no operator's own: the example's plan has that much less room."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


class _Operator:
    def bytes(self):
        return 1000, 101, 64

    def lent(self):
        return 12_000


def test_the_plan_s_memory_is_without_what_is_lent():
    import mlp_stage
    p = mlp_stage.planned(_Operator(), 100.0, 200.0, layers=3)
    assert p.type_mem_bytes.tolist() == [288 * 10**9 - 12_000]
    assert p.param_bytes.tolist() == [500, 1000] * 3 and p.stash_bytes.tolist() == [51, 101] * 3
    assert mlp_stage.planned(_Operator(), 100.0, 200.0, layers=3, memory=20_000).type_mem_bytes.tolist() == [8_000]


@pytest.mark.gpu
def test_lent_is_what_is_neither_parameters_nor_kept(harp):
    """Tensors that the operator holds, by their storage: each is a parameter's, kept for the backward pass, or lent."""
    import torch
    import mlp_stage
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    op = mlp_stage.MlpOperator(ctx, 256, 96, 8)
    own = sum(t.numel() * t.element_size() for t in vars(op).values() if torch.is_tensor(t))
    assert op.lent() + op.bytes()[1] == own
    for need in ((96, 1024, 256), (96, 256, 1024)):
        assert op.ws.numel() >= ops.linear_workspace(ctx, *need).numel(), need
    assert op.ws.numel() >= ops.norm_workspace(ctx, 96, 256).numel()
    ctx.close()
