"""The operators of a pipeline stage's training step: timed cases, plain forms, and what they are in 64 bits.

`linear` is a matrix product with bias, activation and residual in its epilogue, and its gradients; `norm` is the
norm after a block, its gate and residual scale, the residual sum and the norm before the next block, and their
gradients; `adamw` is the optimizer's step over all tensors of some layers, with moments in 32 or in 8 bits.
Sizes follow the planner's workloads: layers of 4,096 and 8,192 channels, cuts of 4,096 tokens, an MLP of four times
the channels.  Each plain form is elementary torch operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
BLOCK = 256                     # elements of one block of an 8-bit state
HYPER = {"lr": 3e-4, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "step": 1000}
DECAY = 0.1                     # of matrices; vectors have none
GRAD_SCALE = 0.5                # what gradients are multiplied by before use (loss scale, clipping)


# ------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token through the first product of a 4,096-channel layer's MLP: serving, bound by the weights
        linear("linear one token", "forward", 1, 4096, 16384, "bf16", act="gelu_tanh", bias=True),
        # a few tokens, ragged sizes: the smallest call, its latency is what counts
        linear("linear seven tokens odd", "forward", 7, 1000, 1037, "f16", act="silu", bias=True, residual=True),
        # a micro-batch of 4,096 tokens through the same product, with what its backward pass needs kept
        linear("linear 4096 tokens", "forward", 4096, 4096, 16384, "bf16", act="gelu_tanh", bias=True, save=True),
        # the second product's gradients: back through the activation, the weights' gradient summed over micro-batches
        linear("linear gradients 4096 tokens", "backward", 4096, 16384, 4096, "bf16", act="gelu_tanh", bias=True,
               accumulate=True),
        # a packed batch of no round length through a narrower layer
        linear("linear gradients 1537 tokens", "backward", 1537, 1224, 4904, "f16", act="relu", bias=True, residual=True),
        # one token between two blocks of an 8,192-channel layer: latency
        norm("norm one token", "forward", 1, 8192, "bf16", "rms", "rms", scale=True),
        # a cut's 4,096 tokens of 8,192 channels, norms on both sides of the block
        norm("norm 4096 tokens", "forward", 4096, 8192, "bf16", "rms", "rms", rows_per_gate=4096, scale=True),
        # its gradients
        norm("norm gradients 4096 tokens", "backward", 4096, 8192, "bf16", "rms", "rms", rows_per_gate=4096, scale=True),
        # a gate for every sample of 257 tokens, layer norms, an odd number of channels in 32 bits
        norm("norm gradients gate a sample", "backward", 2313, 1155, "f32", "layer", "layer", rows_per_gate=257,
             gate_act="sigmoid"),
        # one 4,096-channel layer, 201 million parameters: 16 bytes of weight, gradient, master and moments each
        adamw("adamw a layer", 32, 1, 4096, "bf16"),
        # a 2,048-channel layer, 50 million parameters, moments in 8 bits
        adamw("adamw a layer 8 bits", 8, 1, 2048, "bf16"),
        # the 400 tensors of a small model, most of them a few dozen values long
        adamw("adamw 400 small tensors", 32, 40, 37, "f16"),
    ]


def linear(name, direction, tokens, inputs, outputs, type, act="none", bias=False, residual=False, save=False,
           accumulate=False):
    """accumulate: the weights' gradient is added to one held in 32 bits."""
    return dict(name=name, op="linear", direction=direction, tokens=tokens, inputs=inputs, outputs=outputs, type=type,
                act=act, bias=bias, residual=residual, save=save, accumulate=accumulate)


def norm(name, direction, rows, cols, type, after, before, rows_per_gate=0, gate_act="none", scale=False):
    return dict(name=name, op="norm", direction=direction, rows=rows, cols=cols, type=type, after=after, before=before,
                rows_per_gate=rows_per_gate, gate_act=gate_act, scale=scale)


def adamw(name, state, layers, channels, grad):
    return dict(name=name, op="adamw", state=state, layers=layers, channels=channels, grad=grad)


def draw(rng):
    def size(lo, hi):
        n = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
        return n + 1 if n % 256 == 0 else n      # the listed cases have the round ones

    op = rng.choice(("linear", "linear", "norm", "norm", "adamw"))
    if op == "linear":
        while True:
            tokens, inputs, outputs = size(1, 8192), size(256, 16384), size(256, 16384)
            if rng.random() < 0.6:       # layers' channels are mostly multiples of 64, batches of anything
                inputs, outputs = 64 * (inputs // 64 | 1), 64 * (outputs // 64 | 1)
            if tokens * inputs * outputs <= 4096 * 4096 * 16384 and tokens * inputs * outputs >= 1 << 16:
                break
        direction = rng.choice(("forward", "backward"))
        case = linear("", direction, tokens, inputs, outputs, rng.choice(("bf16", "f16")),
                      act=rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")), bias=rng.random() < 0.7,
                      residual=rng.random() < 0.5, save=direction == "forward" and rng.random() < 0.5,
                      accumulate=direction == "backward" and rng.random() < 0.5)
    elif op == "norm":
        while True:
            rows, cols = size(1, 16384), size(64, 8192)
            if rng.random() < 0.6:
                cols = 64 * (cols // 64 | 1)
            if rows * cols <= 4096 * 8192:
                break
        case = norm("", rng.choice(("forward", "backward")), rows, cols, rng.choice(("bf16", "bf16", "f16", "f32")),
                    rng.choice(("rms", "layer", "none")), rng.choice(("rms", "layer")),
                    rows_per_gate=rng.choice((0, 1, rows, size(1, rows))), gate_act=rng.choice(("none", "sigmoid")),
                    scale=rng.random() < 0.5)
    else:
        channels = size(16, 3800)
        layers = size(1, max(1, min(40, 15_000_000 // (channels * channels))))
        case = adamw("", rng.choice((32, 8)), layers, channels, rng.choice(("bf16", "f16", "f32")))
    del case["name"]
    return case


def work(case):
    if case["op"] == "linear":
        m, k, n, e = case["tokens"], case["inputs"], case["outputs"], 2
        if case["direction"] == "forward":
            count = m * k + n * k + m * n * (1 + case["residual"] + case["save"]) + n * case["bias"]
            return {"bytes": e * count, "flops": 2 * m * n * k}
        count = m * n + n * k + 2 * m * k                       # dY, W, X read, dX written
        count += m * k * ((case["act"] != "none") + case["residual"])
        grad = n * k * (8 if case["accumulate"] else e) + n * case["bias"] * (8 if case["accumulate"] else 4)
        return {"bytes": e * count + grad, "flops": 4 * m * n * k}
    if case["op"] == "norm":
        r, c, e = case["rows"], case["cols"], BYTES[case["type"]]
        gates = -(-r // case["rows_per_gate"]) * c if case["rows_per_gate"] else 0
        vectors = 4 * c * params_of(case)
        if case["direction"] == "forward":
            return {"bytes": e * (4 * r * c + gates) + vectors, "flops": 16 * r * c}
        return {"bytes": e * (6 * r * c + 2 * gates) + 2 * vectors, "flops": 30 * r * c}
    n = sum(sizes(case))
    if case["state"] == 32:
        return {"bytes": n * (BYTES[case["grad"]] + 8 + 16 + 2), "flops": 16 * n}
    # moments in 8 bits are read and written, and their values (16 bits) written for whoever looks at them
    return {"bytes": n * (BYTES[case["grad"]] + 8 + 4 + 2 + 2 + 4), "flops": 60 * n}


def params_of(case):
    """Vectors of cols entries that a norm case has: weights, biases, residual scale."""
    count = {"none": 0, "rms": 1, "layer": 2}
    return count[case["after"]] + count[case["before"]] + case["scale"]


def sizes(case):
    """Elements of every tensor of an adamw case: per layer four square matrices, the two of an MLP of four times the
    channels with their biases, and two norms."""
    c = case["channels"]
    return ([c * c] * 4 + [4 * c * c, 4 * c * c, 4 * c, c, c, c]) * case["layers"]


# ------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"linear": prepare_linear, "norm": prepare_norm, "adamw": prepare_adamw}[case["op"]](case, gen)


def normal(gen, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def context():
    from paper_2509_24859_amd import binding
    return binding.Context(torch.cuda.current_device())


def prepare_linear(case, gen):
    m, k, n, t = case["tokens"], case["inputs"], case["outputs"], TYPES[case["type"]]
    s = {"case": case, "w": normal(gen, (n, k), t, k ** -0.5)}
    if case["direction"] == "forward":
        s["x"] = normal(gen, (m, k), t)
        s["bias"] = normal(gen, (n,), t, 0.5) if case["bias"] else None
        s["residual"] = normal(gen, (m, n), t) if case["residual"] else None
        s["y"] = torch.empty((m, n), dtype=t, device="cuda")
        s["z"] = torch.empty((m, n), dtype=t, device="cuda") if case["save"] else None
    else:
        # x is what the activation of the product before made of z
        s["x"] = normal(gen, (m, k), t)
        s["z"] = normal(gen, (m, k), t) if case["act"] != "none" else None
        s["dy"] = normal(gen, (m, n), t, 0.1)
        s["residual"] = normal(gen, (m, k), t, 0.1) if case["residual"] else None
        s["dx"] = torch.empty((m, k), dtype=t, device="cuda")
        wide = torch.float32 if case["accumulate"] else t
        s["dw"] = normal(gen, (n, k), wide, 0.1) if case["accumulate"] else torch.empty((n, k), dtype=wide, device="cuda")
        s["dbias"] = normal(gen, (n,), torch.float32, 0.1) if case["bias"] else None
    if own:
        from paper_2509_24859_amd import operators
        s["ctx"] = context()
        s["workspace"] = operators.linear_workspace(s["ctx"], m, n, k)
    return s


def prepare_norm(case, gen):
    r, c, t = case["rows"], case["cols"], TYPES[case["type"]]
    # channels of a residual stream differ in size, a few by much
    spread = torch.exp(0.5 * torch.randn(c, generator=gen, device="cuda"))
    spread[:: max(1, c // 4)] *= 20
    s = {"case": case, "y": normal(gen, (r, c), t, 0.7)}
    for at in ("after", "before"):
        kind = case[at]
        s["w_" + at] = 1 + normal(gen, (c,), torch.float32, 0.1) if kind != "none" else None
        s["b_" + at] = normal(gen, (c,), torch.float32, 0.1) if kind == "layer" else None
    s["scale"] = normal(gen, (c,), torch.float32, 0.2) if case["scale"] else None
    groups = -(-r // case["rows_per_gate"]) if case["rows_per_gate"] else 0
    s["gate"] = normal(gen, (groups, c), t) if groups else None
    if case["direction"] == "forward":
        s["x"] = (torch.randn((r, c), generator=gen, device="cuda") * spread).to(t)
        s["h"], s["z"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    else:
        s["h"] = (torch.randn((r, c), generator=gen, device="cuda") * spread).to(t)
        s["dh"], s["dz"] = normal(gen, (r, c), t, 0.01), normal(gen, (r, c), t, 0.1)
        s["dx"], s["dy"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])
        s["dgate"] = torch.empty_like(s["gate"]) if groups else None
        for name in ("w_after", "b_after", "w_before", "b_before", "scale"):
            s["d" + name] = torch.empty(c, dtype=torch.float32, device="cuda") if s[name] is not None else None
    if own:
        from paper_2509_24859_amd import operators
        s["ctx"] = context()
        s["workspace"] = operators.norm_workspace(s["ctx"], r, c, case["rows_per_gate"])
    return s


def prepare_adamw(case, gen):
    """Flat buffers in which every tensor begins at a multiple of 256 elements, as a program keeps its parameters."""
    part = sizes(case)
    blocks = [-(-n // BLOCK) for n in part]
    first = [0]
    for b in blocks:
        first.append(first[-1] + b)
    total = first[-1] * BLOCK
    matrix = [n >= case["channels"] * case["channels"] and n > 4 * case["channels"] for n in part]
    of_block = torch.repeat_interleave(torch.arange(len(part)), torch.tensor(blocks)).cuda()
    inside = torch.tensor(part).cuda()[of_block][:, None] - BLOCK * (
        torch.arange(first[-1], device="cuda") - torch.tensor(first[:-1]).cuda()[of_block])[:, None]
    live = (torch.arange(BLOCK, device="cuda")[None, :] < inside).reshape(-1)       # False between the tensors
    size = torch.exp(torch.randn(len(part), generator=gen, device="cuda") - 6)[of_block]
    p = normal(gen, (total,), torch.float32, 0.02) * live
    grad = ((torch.randn((first[-1], BLOCK), generator=gen, device="cuda") * size[:, None]).reshape(-1) * live).to(
        TYPES[case["grad"]])
    s = {"case": case, "p": p, "grad": grad, "copy": torch.zeros(total, dtype=torch.bfloat16, device="cuda"),
         "decay": torch.tensor([DECAY if x else 0.0 for x in matrix], dtype=torch.float64)[of_block.cpu()].cuda(),
         "grad_scale": torch.full((1,), GRAD_SCALE, dtype=torch.float32, device="cuda"),
         "seed": int(torch.randint(0, 1 << 62, (1,), generator=gen, device="cuda").item())}
    if case["state"] == 32:
        s["m"] = (torch.randn((first[-1], BLOCK), generator=gen, device="cuda") * size[:, None] * 0.3).reshape(-1) * live
        s["v"] = (torch.rand((first[-1], BLOCK), generator=gen, device="cuda") * size[:, None] ** 2).reshape(-1) * live
    else:
        code = (torch.randn(total, generator=gen, device="cuda") * 12 + 100).clamp(0, 127).to(torch.int32)
        sign = torch.randint(0, 2, (total,), generator=gen, device="cuda", dtype=torch.int32) * 128
        s["m"] = ((code + sign) * live).to(torch.uint8)
        s["v"] = ((torch.randn(total, generator=gen, device="cuda") * 16 + 228).clamp(0, 255) * live).to(torch.uint8)
        exponent = torch.floor(torch.log2(size)).to(torch.int32) + 127
        s["m_exp"], s["v_exp"] = exponent.to(torch.uint8), (2 * exponent - 127).clamp(64, 254).to(torch.uint8)
        s["m_seen"], s["v_seen"] = (torch.zeros(total, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if own:
        from paper_2509_24859_amd import operators
        s["ctx"] = context()
        tensors = []
        for i, n in enumerate(part):
            a, b = first[i] * BLOCK, first[i] * BLOCK + n
            t = dict(p=s["p"][a:b], grad=s["grad"][a:b], copy=s["copy"][a:b], m=s["m"][a:b], v=s["v"][a:b],
                     weight_decay=DECAY if matrix[i] else 0.0)
            if case["state"] == 8:
                t |= dict(m_exp=s["m_exp"][first[i]:first[i + 1]], v_exp=s["v_exp"][first[i]:first[i + 1]],
                          m_seen=s["m_seen"][a:b], v_seen=s["v_seen"][a:b])
            tensors.append(t)
        s["plan"] = operators.AdamW(s["ctx"], tensors)
    return s


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if not own:
        return {"linear": plain_linear, "norm": plain_norm, "adamw": plain_adamw}[case["op"]](case, state)
    return {"linear": own_linear, "norm": own_norm, "adamw": own_adamw}[case["op"]](case, state)


def own_linear(case, s):
    from paper_2509_24859_amd import operators
    if case["direction"] == "forward":
        operators.harp_linear_forward(s["ctx"], s["x"], s["w"], s["y"], bias=s["bias"], act=case["act"],
                                      residual=s["residual"], z=s["z"], workspace=s["workspace"])
        return {"y": s["y"]} | ({"z": s["z"]} if case["save"] else {})
    operators.harp_linear_grad_input(s["ctx"], s["dy"], s["w"], s["dx"], act=case["act"], z=s["z"],
                                     residual=s["residual"], workspace=s["workspace"])
    operators.harp_linear_grad_weight(s["ctx"], s["dy"], s["x"], s["dw"], dbias=s["dbias"],
                                      accumulate=case["accumulate"], workspace=s["workspace"])
    return {"dx": s["dx"], "dw": s["dw"]} | ({"dbias": s["dbias"]} if case["bias"] else {})


def own_norm(case, s):
    from paper_2509_24859_amd import operators
    form = dict(after=case["after"], before=case["before"], gate=s["gate"], rows_per_gate=case["rows_per_gate"],
                gate_act=case["gate_act"], scale=s["scale"], w_after=s["w_after"], b_after=s["b_after"],
                w_before=s["w_before"], b_before=s["b_before"], eps=EPS)
    if case["direction"] == "forward":
        operators.harp_norm_forward(s["ctx"], s["x"], s["y"], s["h"], s["z"], **form)
        return {"h": s["h"], "z": s["z"]}
    names = [n for n in ("dgate", "dscale", "dw_after", "db_after", "dw_before", "db_before") if s[n] is not None]
    grads = {n: s[n] for n in names}
    operators.harp_norm_backward(s["ctx"], s["dh"], s["dz"], s["h"], s["y"], s["dx"], s["dy"], **form, **grads,
                                 workspace=s["workspace"])
    return {"dx": s["dx"], "dy": s["dy"]} | grads


def own_adamw(case, s):
    s["plan"].step(**HYPER, grad_scale=s["grad_scale"], seed=s["seed"])
    if case["state"] == 32:
        return {"p": s["p"], "m": s["m"], "v": s["v"], "copy": s["copy"]}
    s["plan"].read_state()
    return {"p": s["p"], "m": s["m_seen"], "v": s["v_seen"], "copy": s["copy"]}


# ------------------------------------------------------------------------------------------------- plain forms, 32 bits
def activation(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        th = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * (c * (1 + 3 * 0.044715 * z * z))
    sg = 1 / (1 + torch.exp(-z))
    return sg * (1 + z * (1 - sg))


def plain_linear(case, s):
    t = TYPES[case["type"]]
    w = s["w"].float()
    if case["direction"] == "forward":
        z = s["x"].float() @ w.t()
        if case["bias"]:
            z = z + s["bias"].float()
        y = activation(z, case["act"])
        if case["residual"]:
            y = y + s["residual"].float()
        return {"y": y.to(t)} | ({"z": z.to(t)} if case["save"] else {})
    dy = s["dy"].float()
    dx = dy @ w
    if case["act"] != "none":
        dx = dx * slope(s["z"].float(), case["act"])
    if case["residual"]:
        dx = dx + s["residual"].float()
    dw = dy.t() @ s["x"].float()
    out = {"dx": dx.to(t)}
    if case["accumulate"]:
        s["dw"].add_(dw)
        out["dw"] = s["dw"]
    else:
        out["dw"] = dw.to(t)
    if case["bias"]:
        if case["accumulate"]:
            s["dbias"].add_(dy.sum(0))
            out["dbias"] = s["dbias"]
        else:
            out["dbias"] = dy.sum(0)
    return out


def normed(v, kind):
    """(normalised rows, 1 / deviation)."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * rstd, rstd


def norm_slope(d, hat, rstd, kind):
    d = d - hat * (d * hat).mean(1, keepdim=True) if kind == "rms" else \
        d - d.mean(1, keepdim=True) - hat * (d * hat).mean(1, keepdim=True)
    return d * rstd


def plain_norm(case, s):
    t, r, per = TYPES[case["type"]], case["rows"], case["rows_per_gate"]
    y = s["y"].float()
    hat_y, rstd_y = (y, None) if case["after"] == "none" else normed(y, case["after"])
    branch = hat_y if s["w_after"] is None else hat_y * s["w_after"]
    if s["b_after"] is not None:
        branch = branch + s["b_after"]
    factor, gate = None, None
    if per:
        g = s["gate"].float()
        gate = 1 / (1 + torch.exp(-g)) if case["gate_act"] == "sigmoid" else g
        gate = gate.repeat_interleave(per, 0)[:r]
        factor = gate
    if case["scale"]:
        factor = s["scale"][None, :] if factor is None else factor * s["scale"]
    if case["direction"] == "forward":
        h = s["x"].float() + (branch if factor is None else branch * factor)
        z = normed(h, case["before"])[0] * s["w_before"]
        if s["b_before"] is not None:
            z = z + s["b_before"]
        return {"h": h.to(t), "z": z.to(t)}
    dz = s["dz"].float()
    hat_h, rstd_h = normed(s["h"].float(), case["before"])
    total = s["dh"].float() + norm_slope(dz * s["w_before"], hat_h, rstd_h, case["before"])
    dt = total if factor is None else total * factor
    d_hat = dt if s["w_after"] is None else dt * s["w_after"]
    dy = d_hat if case["after"] == "none" else norm_slope(d_hat, hat_y, rstd_y, case["after"])
    out = {"dx": total.to(t), "dy": dy.to(t)}
    if per:
        dg = total * branch
        if case["scale"]:
            dg = dg * s["scale"]
        if case["gate_act"] == "sigmoid":
            dg = dg * gate * (1 - gate)
        groups = s["gate"].shape[0]
        dg = torch.nn.functional.pad(dg, (0, 0, 0, groups * per - r)).reshape(groups, per, -1).sum(1)
        out["dgate"] = dg.to(t)
    if case["scale"]:
        out["dscale"] = (total * branch if gate is None else total * branch * gate).sum(0)
    if s["w_after"] is not None:
        out["dw_after"] = (dt * hat_y).sum(0)
    if s["b_after"] is not None:
        out["db_after"] = dt.sum(0)
    out["dw_before"] = (dz * hat_h).sum(0)
    if s["b_before"] is not None:
        out["db_before"] = dz.sum(0)
    return out


def random_bits(count, seed):
    """[count] and [count] integers of 16 bits: a hash of the seed and the element's place, one of 64 bits for two
    elements (splitmix64: Steele, Lea, Flood 2014)."""
    z = torch.arange(-(-count // 2), dtype=torch.int64, device="cuda") * -0x61C8864680B583EB + seed
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * -0x40A7B892E31B1A47
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * -0x6B2FB644ECCEEE15
    z = z ^ ((z >> 31) & ((1 << 33) - 1))
    m = torch.stack((z & 0xFFFF, (z >> 32) & 0xFFFF), 1).reshape(-1)[:count]
    v = torch.stack(((z >> 16) & 0xFFFF, (z >> 48) & 0xFFFF), 1).reshape(-1)[:count]
    return m.to(torch.int32), v.to(torch.int32)


def from_codes(code, exponent, top):
    """What 8-bit codes stand for: `top` is the largest exponent field, 15 for m (with a sign), 31 for v."""
    code = code.to(torch.int32).view(-1, BLOCK)
    sign = 1 - 2 * (code >> 7) if top == 15 else 1
    mag = code & 127 if top == 15 else code
    e, f = mag >> 3, mag & 7
    whole = torch.where(e > 0, (8 + f).long() << torch.clamp(e - 1, min=0), f.long())
    unit = ((exponent.to(torch.int32) - top - 2) << 23).view(torch.float32)
    value = (sign * whole).to(torch.float32) * unit[:, None]
    return torch.where(exponent[:, None] == 255, torch.full_like(value, math.nan), value).view(-1)


def to_codes(x, rnd, top):
    """Codes and block exponents of x: each value goes up with the probability of what is cut off."""
    bits = x.view(-1, BLOCK).view(torch.int32)
    mag = bits & 0x7FFFFFFF
    largest = mag.amax(1)
    exponent = torch.clamp((largest + 0xFFFFF) >> 23, min=64)
    exponent = torch.where(largest >= 0x7F800000, torch.full_like(exponent, 255), torch.clamp(exponent, max=254))
    field = mag >> 23
    whole = (mag & 0x7FFFFF) | torch.where(field > 0, 0x800000, 0)
    rel = torch.clamp(field, min=1) - exponent[:, None] + top
    fixed = torch.where(rel >= 1, ((torch.clamp(rel, min=1) - 1) << 23) + whole, whole >> torch.clamp(1 - rel, 0, 31))
    code = torch.clamp((fixed + (rnd.view(-1, BLOCK) << 4)) >> 20, max=127 if top == 15 else 255)
    code = torch.where(exponent[:, None] == 255, torch.zeros_like(code), code)
    if top == 15:
        code = code | ((bits >> 24) & 128)
    return code.to(torch.uint8).view(-1), exponent.to(torch.uint8)


def plain_adamw(case, s):
    b1, b2, lr = HYPER["beta1"], HYPER["beta2"], HYPER["lr"]
    c1, c2 = 1 - b1 ** HYPER["step"], 1 - b2 ** HYPER["step"]
    g = s["grad"].float() * s["grad_scale"]
    eight = case["state"] == 8
    m, v = (from_codes(s["m"], s["m_exp"], 15), from_codes(s["v"], s["v_exp"], 31)) if eight else (s["m"], s["v"])
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    keep = (1 - lr * s["decay"]).float()
    p = (s["p"].view(-1, BLOCK) * keep[:, None]).view(-1)
    p = p - (lr / c1) * m / (torch.sqrt(v) * (1 / math.sqrt(c2)) + HYPER["eps"])
    s["p"].copy_(p)
    s["copy"].copy_(p)
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {"p": s["p"], "m": s["m"], "v": s["v"], "copy": s["copy"]}
    rm, rv = random_bits(p.numel(), s["seed"])
    for name, x, rnd, top in (("m", m, rm, 15), ("v", v, rv, 31)):
        code, exponent = to_codes(x, rnd, top)
        s[name].copy_(code)
        s[name + "_exp"].copy_(exponent)
        s[name + "_seen"].copy_(from_codes(code, exponent, top))
    return {"p": s["p"], "m": s["m_seen"], "v": s["v_seen"], "copy": s["copy"]}


# ------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    d = {k: x.double() for k, x in s.items() if torch.is_tensor(x) and x.is_floating_point()}
    return {"linear": exact_linear, "norm": exact_norm, "adamw": exact_adamw}[case["op"]](case, s, d)


def exact_act(z, act):
    """The activation and its derivative."""
    if act == "relu":
        on = (z > 0).double()
        return z * on, on
    if act == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":             # (1 + tanh(u)) / 2 is the logistic function of 2 u
        u = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        sg = torch.sigmoid(u)
        return z * sg, sg + z * sg * torch.sigmoid(-u) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * z ** 2)
    if act == "silu":
        sg = torch.sigmoid(z)
        return z * sg, sg + z * sg * torch.sigmoid(-z)
    return z, torch.ones_like(z)


def exact_linear(case, s, d):
    if case["direction"] == "forward":
        z = torch.mm(d["x"], d["w"].t().contiguous())
        z = z + d["bias"] if case["bias"] else z
        y = exact_act(z, case["act"])[0]
        y = y + d["residual"] if case["residual"] else y
        return {"y": y} | ({"z": z} if case["save"] else {})
    dx = torch.mm(d["dy"], d["w"])
    dx = dx * exact_act(d["z"], case["act"])[1] if case["act"] != "none" else dx
    dx = dx + d["residual"] if case["residual"] else dx
    dw = torch.mm(d["dy"].t().contiguous(), d["x"])
    out = {"dx": dx, "dw": dw + d["dw"] if case["accumulate"] else dw}
    if case["bias"]:
        out["dbias"] = d["dy"].sum(0) + (d["dbias"] if case["accumulate"] else 0)
    return out


def exact_norm(case, s, d):
    """The backward pass by differentiation of the forward one."""
    names = ["y", "gate", "scale", "w_after", "b_after", "w_before", "b_before"]
    v = {n: d[n].requires_grad_(case["direction"] == "backward") for n in names if n in d}

    def unit(a, at):
        kind = case[at]
        if kind == "none":
            return a
        a = a - a.mean(dim=1, keepdim=True) if kind == "layer" else a
        a = a / (a.square().mean(dim=1, keepdim=True) + EPS).sqrt()
        return a * v["w_" + at] + v.get("b_" + at, 0)

    branch = unit(v["y"], "after")
    if "gate" in v:
        gate = torch.sigmoid(v["gate"]) if case["gate_act"] == "sigmoid" else v["gate"]
        row = torch.arange(case["rows"], device="cuda") // case["rows_per_gate"]
        branch = branch * gate[row]
    branch = branch * v["scale"] if "scale" in v else branch
    if case["direction"] == "forward":
        h = d["x"] + branch
        return {"h": h, "z": unit(h, "before")}
    h = d["h"].requires_grad_()
    unit(h, "before").backward(d["dz"])
    total = d["dh"] + h.grad
    branch.backward(total)
    out = {"dx": total, "dy": v["y"].grad}
    return out | {"d" + n: v[n].grad for n in names[1:] if n in v}


def exact_adamw(case, s, d):
    b1, b2 = HYPER["beta1"], HYPER["beta2"]
    g = d["grad"] * GRAD_SCALE
    if case["state"] == 8:
        old = {}
        for name, top in (("m", 15), ("v", 31)):
            mag = s[name].long() % 128 if top == 15 else s[name].long()
            e = torch.div(mag, 8, rounding_mode="floor")
            unit = 2.0 ** (s[name + "_exp"].double() - 129 - top).repeat_interleave(BLOCK)
            old[name] = torch.where(e > 0, (8.0 + mag % 8) * 2.0 ** (e - 1).double(), (mag % 8).double()) * unit
        old["m"] = torch.where(s["m"] >= 128, -old["m"], old["m"])
    else:
        old = {"m": d["m"], "v": d["v"]}
    m = old["m"] + (g - old["m"]) * (1 - b1)
    v = old["v"] + (g ** 2 - old["v"]) * (1 - b2)
    up = m / (1 - b1 ** HYPER["step"]) / ((v / (1 - b2 ** HYPER["step"])).sqrt() + HYPER["eps"])
    decay = s["decay"].repeat_interleave(BLOCK)
    p = d["p"] - HYPER["lr"] * (decay * d["p"] + up)
    out = {"p": p, "copy": p}
    if case["state"] == 32:
        return out | {"m": m, "v": v}
    for (name, x, top), rnd in zip((("m", m, 15), ("v", v, 31)), random_bits(p.numel(), s["seed"])):
        a = x.abs().view(-1, BLOCK)
        largest = a.amax(1).clamp(min=2.0 ** -63)
        e = torch.floor(torch.log2(largest))
        e = torch.where(largest > 1.875 * 2.0 ** e, e + 1, e)
        fine = torch.clamp(torch.floor(torch.log2(a.clamp(min=1e-300))), min=(e - top + 1)[:, None])
        step = 2.0 ** (fine - 3)
        q = torch.floor(a / step + rnd.view(-1, BLOCK).double() / 65536) * step
        out[name] = (q * torch.sign(x.view(-1, BLOCK))).view(-1)
    return out
