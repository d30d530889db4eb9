"""A decoder layer as a pipeline stage runs it - attention operator and gated MLP operator - and a plan with both measured rows.

Each operator reads the normed stream a, adds its block to the residual stream h and hands on h' and the next norm's a'.  Forward,
backward over micro-batches and the optimizer's step run with the package's operators; both operators are timed, and layers of them
are planned over two groups of these GPUs.

    python examples/decoder_layer.py                    # 4,096 channels, 4,096 tokens in 2 sequences, 32 heads on 8
    python examples/decoder_layer.py --channels 8192 --heads 64 --kv-heads 8 --bits 8
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

import mlp_stage
from mlp_stage import microseconds
from paper_2509_24859_amd import binding as harp, operators as ops, workloads


class Operator:
    """Weights in bfloat16 for the products, masters, gradients and moments as in mlp_stage, and what the operators have in common:
    y of the block, h' = h + scale * after(y), a' = before(h')."""

    def __init__(self, ctx, channels: int, tokens: int, bits: int, matrices: dict, seed: int):
        self.ctx, self.c, self.n = ctx, channels, tokens
        gen = torch.Generator(device=ctx.device).manual_seed(seed)
        self.master = {k: torch.randn(s, generator=gen, device=ctx.device) * s[1] ** -0.5 for k, s in matrices.items()}
        self.low = {k: p.bfloat16() for k, p in self.master.items()}
        self.master |= {"w_after": torch.ones(channels, device=ctx.device), "w_before": torch.ones(channels, device=ctx.device),
                        "scale": torch.full((channels,), 0.5, device=ctx.device)}
        self.grad = {k: torch.zeros_like(p) for k, p in self.master.items()}
        self.y, self.h, self.a, self.dy, self.dh, self.da = (self.rows(channels) for _ in range(6))
        entries = []
        for k, p in self.master.items():
            t = {"p": p.view(-1), "grad": self.grad[k].view(-1), "weight_decay": 0.1 if p.dim() == 2 else 0.0}
            if k in self.low:
                t["copy"] = self.low[k].view(-1)
            if bits == 8 and p.dim() == 2:
                t |= {m: torch.zeros(p.numel(), dtype=torch.uint8, device=ctx.device) for m in ("m", "v")}
                t |= {m: torch.zeros(-(-p.numel() // ops.ADAMW_BLOCK), dtype=torch.uint8, device=ctx.device) for m in ("m_exp", "v_exp")}
            else:
                t |= {m: torch.zeros(p.numel(), device=ctx.device) for m in ("m", "v")}
            entries.append(t)
        self.optimizer, self.bits, self.steps = ops.AdamW(ctx, entries), bits, 0

    def rows(self, cols: int):
        return torch.empty(self.n, cols, dtype=torch.bfloat16, device=self.ctx.device)

    def workspaces(self, *sizes):
        """What products of these sizes and the norms need; the largest does for all, as they run one after the other."""
        return [ops.linear_workspace(self.ctx, self.n, out, inner) for out, inner in sizes] + [ops.norm_workspace(self.ctx, self.n, self.c)]

    def norm(self, h):
        ops.harp_norm_forward(self.ctx, h, self.y, self.h, self.a, scale=self.master["scale"], w_after=self.master["w_after"],
                              w_before=self.master["w_before"])
        return self.h, self.a

    def norm_back(self, dh, da, first):
        m, g = self.master, self.grad
        ops.harp_norm_backward(self.ctx, dh, da, self.h, self.y, self.dh, self.dy, scale=m["scale"], w_after=m["w_after"],
                               w_before=m["w_before"], dscale=g["scale"], dw_after=g["w_after"], dw_before=g["w_before"],
                               accumulate=not first, workspace=self.ws)

    def step(self, lr: float):
        self.steps += 1
        self.optimizer.step(lr, self.steps, seed=self.steps)

    def bytes(self):
        """(parameters with gradient, master and moments; kept per micro-batch; across the cut behind it)."""
        count = sum(p.numel() for p in self.master.values())
        return count * (2 + 4 + 4 + 8 * self.bits // 32), self.kept + 3 * 2 * self.n * self.c, 2 * 2 * self.n * self.c


class Attention(Operator):
    """q, k, v of a, rotary positions, causal attention within the sequences, the product behind it."""

    def __init__(self, ctx, channels, tokens, heads, kv_heads, sequences=1, bits=32, seed=0):
        self.heads, self.kv, self.d = heads, kv_heads, channels // heads
        wide = (heads + 2 * kv_heads) * self.d
        super().__init__(ctx, channels, tokens, bits, {"qkv": (wide, channels), "out": (channels, heads * self.d)}, seed)
        self.qkv, self.dqkv, self.o, self.do = self.rows(wide), self.rows(wide), self.rows(heads * self.d), self.rows(heads * self.d)
        self.lse = torch.empty(heads, tokens, device=ctx.device)
        self.sequences = sequences
        self.frequencies, _ = ops.rotary_frequencies(ctx, self.d)
        self.ws = max(self.workspaces((wide, channels), (channels, heads * self.d))
                      + [ops.attention_workspace(ctx, tokens, tokens, sequences, heads, kv_heads, self.d)], key=lambda w: w.numel())
        self.kept = 2 * tokens * (wide + heads * self.d) + 4 * heads * tokens

    def parts(self, qkv):
        """Queries, keys and values as heads of the projection's rows."""
        x = qkv.view(self.n, -1, self.d)
        return x[:, :self.heads], x[:, self.heads:self.heads + self.kv], x[:, self.heads + self.kv:]

    def turn(self, qkv, inverse=False):
        turned = qkv.view(self.n, -1, self.d)[:, :self.heads + self.kv]
        ops.harp_rotary(self.ctx, turned, turned, self.frequencies, period=self.n // self.sequences, inverse=inverse)

    def forward(self, h, a):
        ops.harp_linear_forward(self.ctx, a, self.low["qkv"], self.qkv, workspace=self.ws)
        self.turn(self.qkv)
        ops.harp_attention_forward(self.ctx, *self.parts(self.qkv), self.o.view(self.n, self.heads, self.d), lse=self.lse, batch=self.sequences,
                                   causal=True, workspace=self.ws)
        ops.harp_linear_forward(self.ctx, self.o, self.low["out"], self.y, workspace=self.ws)
        return self.norm(h)

    def backward(self, a, dh, da, first: bool):
        g, more = self.grad, dict(accumulate=not first, workspace=self.ws)
        self.norm_back(dh, da, first)
        ops.harp_linear_grad_weight(self.ctx, self.dy, self.o, g["out"], **more)
        ops.harp_linear_grad_input(self.ctx, self.dy, self.low["out"], self.do, workspace=self.ws)
        heads = (self.n, self.heads, self.d)
        ops.harp_attention_backward(self.ctx, *self.parts(self.qkv), self.o.view(heads), self.lse, self.do.view(heads), *self.parts(self.dqkv),
                                    batch=self.sequences, causal=True, workspace=self.ws)
        self.turn(self.dqkv, inverse=True)
        ops.harp_linear_grad_weight(self.ctx, self.dqkv, a, g["qkv"], **more)
        ops.harp_linear_grad_input(self.ctx, self.dqkv, self.low["qkv"], self.da, workspace=self.ws)
        return self.dh, self.da


class GatedMlp(Operator):
    """y = W2 (silu(Wg a) * Wu a), the gate's and the other's rows in one matrix."""

    def __init__(self, ctx, channels, tokens, width, bits=32, seed=0):
        super().__init__(ctx, channels, tokens, bits, {"up": (2 * width, channels), "down": (channels, width)}, seed)
        self.u, self.z, self.dz = self.rows(width), self.rows(2 * width), self.rows(2 * width)
        self.ws = max(self.workspaces((2 * width, channels), (channels, width)) + [ops.gated_workspace(ctx, tokens, width, channels)],
                      key=lambda w: w.numel())
        self.kept = 2 * tokens * 2 * width

    def forward(self, h, a):
        ops.harp_gated_forward(self.ctx, a, self.low["up"], self.u, act="silu", z=self.z, workspace=self.ws)
        ops.harp_linear_forward(self.ctx, self.u, self.low["down"], self.y, workspace=self.ws)
        return self.norm(h)

    def backward(self, a, dh, da, first: bool):
        g, more = self.grad, dict(accumulate=not first, workspace=self.ws)
        self.norm_back(dh, da, first)
        # u is made again of z on the way: it need not be kept
        ops.harp_gated_grad(self.ctx, self.dy, self.low["down"], self.z, self.dz, act="silu", h=self.u, workspace=self.ws)
        ops.harp_linear_grad_weight(self.ctx, self.dy, self.u, g["down"], **more)
        ops.harp_linear_grad_weight(self.ctx, self.dz, a, g["up"], **more)
        ops.harp_linear_grad_input(self.ctx, self.dz, self.low["up"], self.da, workspace=self.ws)
        return self.dh, self.da


def problem(rows, layers: int, memory=288 * mlp_stage.GB) -> workloads.Problem:
    """`layers` layers of the attention's and the MLP's measured (forward us, backward us, (parameters, kept, cut)), on the two groups of
    mlp_stage."""
    p = mlp_stage.problem(1, 1, (0, 0, rows[0][2][2]), layers, memory)
    of = lambda f: np.array([max(1, int(np.ceil(f(r)))) for r in rows] * layers, dtype=np.int64)  # noqa: E731
    p.fwd_us, p.bwd_us = of(lambda r: r[0])[None, :], of(lambda r: r[1])[None, :]
    p.param_bytes, p.stash_bytes = of(lambda r: r[2][0]), of(lambda r: r[2][1])
    return p


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("channels", 4096), ("tokens", 4096), ("sequences", 2), ("heads", 32), ("kv-heads", 8), ("layers", 80)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args()
    ctx = harp.Context(0)
    rows = []
    for name in ("attention", "gated MLP"):
        op = (Attention(ctx, a.channels, a.tokens, a.heads, a.kv_heads, a.sequences, a.bits) if name == "attention"
              else GatedMlp(ctx, a.channels, a.tokens, 3 * a.channels, a.bits))
        h, dh = (torch.randn(a.tokens, a.channels, device=ctx.device).bfloat16() for _ in range(2))
        forward = microseconds(lambda: op.forward(h, h))
        backward = microseconds(lambda: op.backward(h, dh, dh, first=False))
        print("%s operator of %d channels, %d tokens: forward %.0f us, backward %.0f us, optimizer step %.0f us"
              % (name, a.channels, a.tokens, forward, backward, microseconds(lambda: op.step(0.0))))
        rows.append((forward, backward, op.bytes()))
    print("plan of %d layers on 2 x 8 GPUs: %s" % (a.layers, mlp_stage.plan(ctx, problem(rows, a.layers)) or "none fits"))
    ctx.close()


if __name__ == "__main__":
    main()
