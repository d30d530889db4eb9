"""Moments in 8 bits of elements that are small beside their block's largest.

A block's codes of v end 2^33 below its largest value, those of m 2^17 below.  An element whose gradient is 2^-r of the
block's steady one has, after its first gradient, v = 0.001 2^-2r of the largest: below the last code from r = 12 on, where
m = 0.1 2^-r still has one.
"""
import pytest

BLOCK = 256
LR = 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("after", [0.0, 2.0 ** -30], ids=["then_nothing", "then_next_to_nothing"])
@pytest.mark.parametrize("r", [8, 10, 12, 13, 14, 15, 18, 22])
def test_a_gradient_that_stops_moves_a_weight_no_further_than_a_first_step(harp, r, after):
    """Blocks whose first element has gradient, m and v of one throughout; the others begin at zero, get 2^-r once and then
    `after`.  The formula's steps are at most 0.1 / sqrt(0.001) = 3.2 lr and fall.  A code of m is less than one step of codes
    off: m is at most 4 units of 2^-17 where it is not above the formula's by more than a fifth, and a v that is rounded
    takes at most an eighth off its value or is at least the last code, 2^-33.  So no step is above 6 lr."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    blocks = 64
    n = blocks * BLOCK
    first = torch.arange(n, device="cuda") % BLOCK == 0
    t = {"p": torch.zeros(n, device="cuda"), "grad": torch.empty(n, device="cuda")}
    # code 15 8 is (8 + 0) 2^14 2^(127 - 144) = 1, of v 31 8 likewise
    t["m"] = torch.where(first, 15 * 8, 0).to(torch.uint8)
    t["v"] = torch.where(first, 31 * 8, 0).to(torch.uint8)
    t["m_exp"], t["v_exp"] = (torch.full((blocks,), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    t["m_seen"], t["v_seen"] = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    plan = ops.AdamW(ctx, [t])
    for k in range(6):
        t["grad"].copy_(torch.where(first, 1.0, 2.0 ** -r if k == 0 else after))
        old = t["p"].clone()
        plan.step(LR, 1_000_000 + k, seed=77 + k)
        assert (t["p"] - old).abs().max().item() <= 6 * LR, (k, (t["p"] - old).abs().max().item() / LR)
        plan.read_state()
        assert (t["v_seen"] > 0).all()
    ctx.close()


@pytest.mark.gpu
def test_what_is_zero_stays_zero(harp):
    """Elements that never had a gradient keep zeros and their weights beside others of any size."""
    import torch
    from paper_2509_24859_amd import operators as ops
    ctx = harp.Context(0)
    n = 3 * BLOCK + 17
    some = torch.arange(n, device="cuda") % 3 == 0
    t = {"p": torch.ones(n, device="cuda"), "grad": torch.where(some, torch.randn(n, device="cuda"), 0.0)}
    for name in ("m", "v"):
        t[name] = torch.zeros(n, dtype=torch.uint8, device="cuda")
        t[name + "_exp"] = torch.zeros(-(-n // BLOCK), dtype=torch.uint8, device="cuda")
    plan = ops.AdamW(ctx, [t])
    for k in range(5):
        plan.step(LR, k + 1, seed=k)
    assert (t["m"][~some] == 0).all() and (t["v"][~some] == 0).all() and (t["p"][~some] == 1).all()
    assert (t["v"][some] != 0).all()
    ctx.close()
