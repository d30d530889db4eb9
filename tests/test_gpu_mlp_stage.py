"""The example that runs the operators together: its gradients, its training, its row in a plan."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _block(v, h, a):
    """The operator in 64 bits, with torch's differentiation."""
    import torch
    z1 = a @ v["w1"].t() + v["b1"]
    u = 0.5 * z1 * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (z1 + 0.044715 * z1 ** 3)))
    y = u @ v["w2"].t() + v["b2"]
    norm = lambda x, w: x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * w  # noqa: E731
    h = h + v["scale"] * norm(y, v["w_after"])
    return h, norm(h, v["w_before"])


@pytest.mark.gpu
def test_gradients_of_the_whole_operator(harp):
    """Tensors of 16 bits lie between the operators: each is off by half a unit of 2^-8, five in a chain, so the results
    are within 5 x 2^-8 of their norm, and a wrong factor or a missing term is far outside."""
    import torch
    import mlp_stage
    ctx = harp.Context(0)
    op = mlp_stage.MlpOperator(ctx, 128, 96, 32)
    h, dh, da = (torch.randn(96, 128, device="cuda").bfloat16() for _ in range(3))
    a = torch.randn(96, 128, device="cuda").bfloat16()
    for k in range(2):                                    # two micro-batches: sums of two
        got_h, got_a = op.forward(h, a)
        out_h, out_a = got_h.clone(), got_a.clone()
        dx, dz = op.backward(a, dh, da, first=k == 0)
    v = {k: (op.low[k] if k in op.low else op.master[k]).double().cpu().requires_grad_() for k in op.NAMES}
    H, A = (t.double().cpu().requires_grad_() for t in (h, a))
    want_h, want_a = _block(v, H, A)
    ((want_h * dh.double().cpu()).sum() + (want_a * da.double().cpu()).sum()).backward()
    pairs = [("h", out_h, want_h, 1), ("a", out_a, want_a, 1), ("dh", dx, H.grad, 1), ("da", dz, A.grad, 1)]
    pairs += [("d" + k, op.grad[k], v[k].grad, 2) for k in op.NAMES]
    for name, got, want, times in pairs:
        off = (got.double().cpu() - times * want).norm() / (times * want).norm()
        assert off < 5 * 2.0 ** -8, (name, off.item())
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_training_lowers_the_loss(harp, bits):
    import mlp_stage
    ctx = harp.Context(0)
    losses = mlp_stage.train(mlp_stage.MlpOperator(ctx, 256, 160, bits), 30)
    assert all(np.isfinite(losses)) and losses[-1] < 0.8 * losses[0], losses
    ctx.close()


@pytest.mark.gpu
def test_a_measured_row_is_planned(harp):
    import mlp_stage
    ctx = harp.Context(0)
    best = {}
    for bits in (32, 8):
        op = mlp_stage.MlpOperator(ctx, 256, 64, bits)
        params, kept, cut = op.bytes()
        assert params == sum(p.numel() for p in op.master.values()) * (18 if bits == 32 else 12)
        # 20 layers; a device has room for an eighth of the 32-bit states and a little
        memory = int(20 * 1.5 * sum(p.numel() for p in op.master.values()) * 18 / 8) + 40 * kept
        best[bits] = mlp_stage.plan(ctx, mlp_stage.problem(100.0, 200.0, (params, kept, cut), layers=20, memory=memory))
    assert best[8] is not None and best[8]["cuts"][-1] == 40
    assert best[32] is None or best[8]["iteration_us"] <= best[32]["iteration_us"]
    ctx.close()


def test_the_problem_of_a_row():
    import mlp_stage
    p = mlp_stage.problem(100.4, 201.0, (1000, 101, 64), layers=3, memory=12345)
    assert p.L == 6 and p.fwd_us.tolist() == [[51, 101] * 3] and p.bwd_us.tolist() == [[101, 201] * 3]
    assert p.param_bytes.tolist() == [500, 1000] * 3 and p.stash_bytes.tolist() == [51, 101] * 3
    assert p.act_bytes.tolist() == [64] * 6 and p.type_mem_bytes.tolist() == [12345] and p.bw[0, 1] == p.bw[1, 0] == 3125
