"""One MLP operator of a pipeline stage on this GPU, and a plan made with its measured row.

The planner takes an operator's forward and backward time and its bytes as given.  Here the MLP operator of a transformer
layer runs with the package's operators as a training step would run it - forward, backward summed over micro-batches,
optimizer step -, is timed, and the row is planned with: 8-bit optimizer states change what a device has room for.

    python examples/mlp_stage.py                    # 4,096 channels, 4,096 tokens
    python examples/mlp_stage.py --bits 8 --channels 8192
"""
from __future__ import annotations

import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

from paper_2509_24859_amd import binding as harp, operators as ops, workloads

GB = 10**9


class MlpOperator:
    """a -> y = W2 gelu(W1 a + b1) + b2,  h' = h + scale * after(y),  a' = before(h'): the block with the norm behind it,
    the residual sum, and the norm that the next block reads.  Weights in bfloat16 for the products, masters, gradients
    and sums in 32 bits, moments in 32 or 8 bits."""

    NAMES = ("w1", "b1", "w2", "b2", "w_after", "w_before", "scale")

    def __init__(self, ctx, channels: int, tokens: int, bits: int = 32, wide: int = 4, seed: int = 0):
        self.ctx, self.c, self.n, self.f, self.bits = ctx, channels, tokens, wide * channels, bits
        d, gen = ctx.device, torch.Generator(device=ctx.device).manual_seed(seed)
        c, f = self.c, self.f

        def normal(*shape, std):
            return torch.randn(shape, generator=gen, device=d) * std

        self.master = {"w1": normal(f, c, std=c ** -0.5), "b1": normal(f, std=0.02), "w2": normal(c, f, std=f ** -0.5),
                       "b2": normal(c, std=0.02), "w_after": torch.ones(c, device=d), "w_before": torch.ones(c, device=d),
                       "scale": torch.full((c,), 0.5, device=d)}
        self.grad = {k: torch.zeros_like(p) for k, p in self.master.items()}
        self.low = {k: self.master[k].bfloat16() for k in ("w1", "b1", "w2", "b2")}       # what the products read
        b = dict(dtype=torch.bfloat16, device=d)
        n = tokens
        self.z1, self.u, self.dz1 = (torch.empty(n, f, **b) for _ in range(3))
        self.y, self.h, self.a, self.dy, self.dh, self.da = (torch.empty(n, c, **b) for _ in range(6))
        # one workspace for all, as they run one after the other
        self.ws = max((ops.linear_workspace(ctx, n, f, c), ops.linear_workspace(ctx, n, c, f), ops.norm_workspace(ctx, n, c)),
                      key=lambda w: w.numel())
        self.steps = 0
        entries = []
        for k, p in self.master.items():
            t = {"p": p.view(-1), "grad": self.grad[k].view(-1), "weight_decay": 0.1 if p.dim() == 2 else 0.0}
            if k in self.low:
                t["copy"] = self.low[k].view(-1)
            if bits == 8 and p.dim() == 2:            # vectors are few: theirs stay in 32 bits
                blocks = -(-p.numel() // ops.ADAMW_BLOCK)
                t |= {m: torch.zeros(p.numel(), dtype=torch.uint8, device=d) for m in ("m", "v")}
                t |= {m: torch.zeros(blocks, dtype=torch.uint8, device=d) for m in ("m_exp", "v_exp")}
            else:
                t |= {m: torch.zeros(p.numel(), device=d) for m in ("m", "v")}
            entries.append(t)
        self.optimizer = ops.AdamW(ctx, entries)

    def forward(self, h, a):
        """h' and a' of the residual stream h and the normed input a; they hold until the next call."""
        ops.harp_linear_forward(self.ctx, a, self.low["w1"], self.u, bias=self.low["b1"], act="gelu_tanh", z=self.z1,
                                workspace=self.ws)
        ops.harp_linear_forward(self.ctx, self.u, self.low["w2"], self.y, bias=self.low["b2"], workspace=self.ws)
        ops.harp_norm_forward(self.ctx, h, self.y, self.h, self.a, after="rms", before="rms", scale=self.master["scale"],
                              w_after=self.master["w_after"], w_before=self.master["w_before"])
        return self.h, self.a

    def backward(self, a, dh, da, first: bool):
        """Gradients of h and a, given those of h' and a' (dh may be None); the weights' are added up over the
        micro-batches of a step, from the first on.  The residual stream's is the same tensor in and out."""
        m, g = self.master, self.grad
        ops.harp_norm_backward(self.ctx, dh, da, self.h, self.y, self.dh, self.dy, after="rms", before="rms", scale=m["scale"],
                               w_after=m["w_after"], w_before=m["w_before"], dscale=g["scale"], dw_after=g["w_after"],
                               dw_before=g["w_before"], accumulate=not first, workspace=self.ws)
        ops.harp_linear_grad_weight(self.ctx, self.dy, self.u, g["w2"], dbias=g["b2"], accumulate=not first, workspace=self.ws)
        ops.harp_linear_grad_input(self.ctx, self.dy, self.low["w2"], self.dz1, act="gelu_tanh", z=self.z1, workspace=self.ws)
        ops.harp_linear_grad_weight(self.ctx, self.dz1, a, g["w1"], dbias=g["b1"], accumulate=not first, workspace=self.ws)
        ops.harp_linear_grad_input(self.ctx, self.dz1, self.low["w1"], self.da, workspace=self.ws)
        return self.dh, self.da

    def step(self, lr: float):
        self.steps += 1
        self.optimizer.step(lr, self.steps, seed=self.steps)

    def bytes(self):
        """(parameters with gradient, master and moments; kept per micro-batch; across the cut behind it)."""
        count = sum(p.numel() for p in self.master.values())
        kept = 2 * self.n * (2 * self.f + 3 * self.c)                  # z1, u; y, h, a
        return count * (2 + 4 + 4 + 8 * self.bits // 32), kept, 2 * 2 * self.n * self.c

    def lent(self):
        """Bytes that the operators of a device use one after the other, however many they are: the workspace, and the
        gradients on their way back."""
        return sum(t.numel() * t.element_size() for t in (self.ws, self.dz1, self.dy, self.dh, self.da))


def microseconds(call, repeat: int = 10) -> float:
    for _ in range(3):
        call()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(repeat):
        call()
    end.record()
    end.synchronize()
    return begin.elapsed_time(end) * 1000 / repeat


def train(op: MlpOperator, steps: int, micro: int = 2, lr: float = 1e-3, seed: int = 1):
    """Losses of a regression of a' onto fixed targets, the gradients of `micro` micro-batches added up a step."""
    gen = torch.Generator(device=op.ctx.device).manual_seed(seed)
    data = []
    for _ in range(micro):
        h = torch.randn(op.n, op.c, generator=gen, device=op.ctx.device).bfloat16()
        a = torch.empty_like(h)
        ops.harp_norm_forward(op.ctx, h, None, None, a, before="rms")
        data.append((h, a, torch.randn(op.n, op.c, generator=gen, device=op.ctx.device)))
    losses = []
    for _ in range(steps):
        total = 0.0
        for k, (h, a, target) in enumerate(data):
            _, out = op.forward(h, a)
            off = out.float() - target
            total += 0.5 * off.square().mean().item() / micro
            op.backward(a, None, (off / (off.numel() * micro) * 1024).bfloat16(), first=k == 0)
        op.step(lr)                                   # AdamW does not mind the gradients' scale of 1,024
        losses.append(total)
    return losses


def problem(forward_us: float, backward_us: float, sizes, layers: int = 80, memory=288 * GB) -> workloads.Problem:
    """`layers` layers of an attention operator (half an MLP's time and bytes, as in the fine-grained workload) and the
    measured MLP operator, on two groups of eight of these GPUs, 400 GB/s inside and 25 Gb/s between."""
    params, kept, cut = sizes

    def row(x):
        return np.array([[max(1, math.ceil(x / 2)), max(1, math.ceil(x))]] * layers, dtype=np.int64).reshape(-1)

    bw = np.full((2, 2), 25 * 125, dtype=np.int64)
    np.fill_diagonal(bw, 400 * 1000)
    return workloads.Problem(
        L=2 * layers, T=1, G=2, M=64, ar_count=4, tp_degrees=np.array([1, 2, 4, 8], dtype=np.int32),
        fwd_us=row(forward_us)[None, :], bwd_us=row(backward_us)[None, :], param_bytes=row(params), stash_bytes=row(kept),
        act_bytes=np.full(2 * layers, cut, dtype=np.int64), group_type=np.zeros(2, dtype=np.int32),
        group_ndev=np.full(2, 8, dtype=np.int32), type_mem_bytes=np.array([memory], dtype=np.int64), bw=bw)


def planned(op: MlpOperator, forward_us: float, backward_us: float, layers: int = 80, memory=288 * GB) -> workloads.Problem:
    """problem() of this operator on devices that have lent what its calls use in turn."""
    return problem(forward_us, backward_us, op.bytes(), layers, memory - op.lent())


def plan(ctx, p: workloads.Problem):
    """The best plan over both orders of the groups and all stage counts, or None."""
    orders = workloads.orderings_from_lists([(S, list(o)) for S in range(2, 17) for o in ((0, 1), (1, 0))], S_max=16)
    plans, _ = harp.plan_mesh_h1f1b_sweep(ctx, p, orders)
    ok = plans.status == harp.CAND_OK
    if not ok.any():
        return None
    best = int(np.flatnonzero(ok)[plans.iter_time[ok].argmin()])
    S = int(orders.ord_S[best])
    return {"iteration_us": int(plans.iter_time[best]), "stages": S, "cuts": plans.splits[best, :S + 1].tolist(),
            "devices": plans.stage_tp[best, :S].tolist(), "warmup": plans.warmup[best, :S].tolist()}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--channels", type=int, default=4096)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32)
    ap.add_argument("--layers", type=int, default=80)
    a = ap.parse_args()
    ctx = harp.Context(0)
    op = MlpOperator(ctx, a.channels, a.tokens, a.bits)
    losses = train(op, 5)
    print("loss of 5 steps: " + ", ".join("%.4f" % x for x in losses))
    h = torch.randn(a.tokens, a.channels, device=ctx.device).bfloat16()
    dh = torch.randn_like(h)
    forward = microseconds(lambda: op.forward(h, h))
    backward = microseconds(lambda: op.backward(h, dh, dh, first=False))
    step = microseconds(lambda: op.step(0.0))
    sizes = op.bytes()
    print("MLP operator of %d channels, %d tokens: forward %.0f us, backward %.0f us, optimizer step %.0f us"
          % (a.channels, a.tokens, forward, backward, step))
    print("%.2f GB of weights, gradients, masters and moments (%d bits), %.2f GB kept per micro-batch, %.0f MB across a cut, "
          "%.2f GB lent by the device" % (sizes[0] / 1e9, a.bits, sizes[1] / 1e9, sizes[2] / 1e6, op.lent() / 1e9))
    p = planned(op, forward, backward, a.layers)
    print("plan of %d layers on 2 x 8 GPUs: %s" % (a.layers, plan(ctx, p) or "none fits"))
    ctx.close()


if __name__ == "__main__":
    main()
