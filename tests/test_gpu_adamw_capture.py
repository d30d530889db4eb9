"""AdamW and graphs: what a replay repeats, and that a plan is not made during a capture."""
import pytest

HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8)


def _entries(torch, bits, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = 5000
    t = {"p": torch.randn(n, generator=gen, device="cuda"), "grad": torch.randn(n, generator=gen, device="cuda")}
    if bits == 32:
        t |= {name: torch.zeros(n, device="cuda") for name in ("m", "v")}
    else:
        t |= {name: torch.zeros(n, dtype=torch.uint8, device="cuda") for name in ("m", "v")}
        t |= {name: torch.zeros(-(-n // 256), dtype=torch.uint8, device="cuda") for name in ("m_exp", "v_exp")}
    return t


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_replay_is_the_captured_step_again(harp, bits):
    """lr, step and seed are the captured call's; gradients, grad_scale and skip are read at the replay."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    a, b = _entries(torch, bits, 3), _entries(torch, bits, 3)
    scale, skip = torch.ones(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    plan, other = ops.AdamW(ctx, [a]), ops.AdamW(ctx, [b])
    how = dict(HYPER, lr=1e-3, step=4, seed=99, grad_scale=scale, skip=skip)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.step(**how)
    for k in range(4):
        a["grad"].mul_(0.5)
        b["grad"].mul_(0.5)
        scale.fill_(1.0 + k)
        skip.fill_(int(k == 2))
        graph.replay()
        torch.cuda.synchronize()
        other.step(**how)
        torch.cuda.synchronize()
        assert all(torch.equal(a[name], b[name]) for name in a), k
    ctx.close()


@pytest.mark.gpu
def test_no_plan_during_a_capture(harp):
    """It is written from the host and waited for: refused, and the capture goes on."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    t, x = _entries(torch, 32, 5), torch.zeros(16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1)
        with pytest.raises(harp.HarpError) as err:
            ops.AdamW(ctx, [t])
        x.add_(1)
    assert err.value.code == harp.ERR_INVALID_ARG and "captur" in str(err.value)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert (x == 2 * (k + 1)).all()
    ops.AdamW(ctx, [t]).step(1e-3, 1)                     # and afterwards it is made
    torch.cuda.synchronize()
    assert torch.isfinite(t["p"]).all()
    ctx.close()
