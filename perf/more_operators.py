"""The operators of a layer beyond products, norms and the optimizer: timed cases, plain forms, and what they are in 64 bits.

`rotary` turns pairs of channels by an angle that grows with the position; `attention` is softmax attention of packed or padded
sequences to keys of the same or of another length, and its gradients; `gated` is the first half of a gated feed-forward
block - two projections, an activation and a product - and its gradients.  Sizes follow the planner's workloads: layers of 4,096
and 8,192 channels in heads of 128, cuts of 4,096 tokens.  Each plain form is elementary torch operations in 32 bits
(angles in 64), rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BASE = 10000.0


# ------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # queries and keys of one new token of an 8,192-channel layer: the smallest call, its latency is what counts
        rotary("rotary one token", "forward", 1, 72, 128, 128, "bf16", "interleaved", far=131072),
        # a cut's 4,096 tokens: the 40 heads of queries and keys out of a projection's 48, context stretched eight times by parts
        rotary("rotary 4096 tokens", "forward", 4096, 40, 128, 128, "bf16", "half", skip=8, scaling="by_parts", far=65536),
        # gradients of a packed batch in 32 bits, three quarters of each head turned
        rotary("rotary gradients part of head", "backward", 2313, 12, 96, 72, "f32", "interleaved", scaling="linear", far=4000),
        # one new token for each of 16 sequences, caches of up to 16,384 tokens: serving, bound by reading keys and values
        attention("attention one token", "forward", 16, 1, 16384, 32, 8, 128, "bf16", ragged=True, padded=True),
        # a 4,096-channel layer's causal self attention over a cut of 4,096 tokens, with what its backward pass needs
        attention("attention 4096 tokens", "forward", 1, 4096, 4096, 32, 32, 128, "bf16", causal=True, save=True),
        # its gradients
        attention("attention gradients 4096 tokens", "backward", 1, 4096, 4096, 32, 32, 128, "bf16", causal=True),
        # a decoder's packed sentences over an encoder's padded states
        attention("attention encoder states", "forward", 6, 311, 1500, 16, 16, 64, "f16", ragged=True, padded=True, save=True),
        # gradients of the same with grouped heads of 80, packed on both sides
        attention("attention gradients encoder states", "backward", 5, 777, 450, 12, 4, 80, "f16", ragged=True),
        # one token through a gated block of a 4,096-channel layer: bound by the weights
        gated("gated one token", "forward", 1, 4096, 12288, "bf16", "silu"),
        # a micro-batch of 4,096 tokens, with what its backward pass needs
        gated("gated 4096 tokens", "forward", 4096, 4096, 12288, "bf16", "silu", save=True),
        # back through the second product and the gate, then the input's and both projections' gradients
        gated("gated gradients 4096 tokens", "backward", 4096, 4096, 12288, "bf16", "silu"),
        # a packed batch of no round length through a narrower layer
        gated("gated gradients 1537 tokens", "backward", 1537, 1224, 3268, "f16", "gelu_tanh"),
    ]


def rotary(name, direction, tokens, heads, head, turned, type, layout, skip=0, scaling="none", far=0):
    """skip: heads of a token that lie behind those turned; far: positions are up to this."""
    return dict(name=name, op="rotary", direction=direction, tokens=tokens, heads=heads, head=head, turned=turned, type=type,
                layout=layout, skip=skip, scaling=scaling, far=far)


def attention(name, direction, batch, q_len, k_len, heads, kv_heads, head, type, causal=False, ragged=False, padded=False,
              save=False):
    """q_len, k_len: of the longest sequence.  ragged: others are shorter; padded: keys lie k_len apart, of which a
    sequence uses its count; save: the rows' log-sums are kept."""
    return dict(name=name, op="attention", direction=direction, batch=batch, q_len=q_len, k_len=k_len, heads=heads,
                kv_heads=kv_heads, head=head, type=type, causal=causal, ragged=ragged, padded=padded, save=save)


def gated(name, direction, tokens, channels, width, type, act, bias=False, save=False):
    return dict(name=name, op="gated", direction=direction, tokens=tokens, channels=channels, width=width, type=type, act=act,
                bias=bias, save=save)


def draw(rng):
    def size(lo, hi):
        n = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
        return n + 1 if n % 256 == 0 else n      # the listed cases have the round ones

    op = rng.choice(("rotary", "attention", "attention", "attention", "gated", "gated"))
    type16 = rng.choice(("bf16", "f16"))
    if op == "rotary":
        head = rng.choice((32, 64, 80, 96, 128, 128, 256))
        turned = rng.choice((head, head, head // 2, head // 4 * 2 - 6))
        while True:
            tokens, heads = size(1, 16384), size(1, 80)
            if tokens * heads * head <= 4096 * 40 * 128:
                break
        case = rotary("", rng.choice(("forward", "backward")), tokens, heads, head, turned, rng.choice(("bf16", "f16", "f32")),
                      rng.choice(("half", "interleaved")), skip=rng.choice((0, 0, 1, 8)),
                      scaling=rng.choice(("none", "linear", "ntk", "by_parts")), far=size(100, 1000000))
    elif op == "attention":
        direction, causal = rng.choice(("forward", "forward", "backward")), rng.random() < 0.4
        kv_heads, group, head = rng.choice((1, 2, 3, 4, 8, 16)), rng.choice((1, 1, 2, 3, 4, 8)), rng.choice((32, 64, 72, 80, 96, 128, 128))
        while True:
            batch, q_len, k_len = size(1, 16), 1 if rng.random() < 0.25 else size(1, 4096), size(1, 16384)
            k_len = max(q_len, k_len) if causal else k_len
            work_of = batch * q_len * k_len * kv_heads * group * head
            cache = batch * k_len * kv_heads * head
            if work_of <= (1 << 35) * (1 if direction == "backward" else 2) and cache <= 1 << 28 and work_of >= 1 << 16:
                break
        case = attention("", direction, batch, q_len, k_len, kv_heads * group, kv_heads, head, type16, causal=causal,
                         ragged=rng.random() < 0.7, padded=rng.random() < 0.5, save=direction == "forward" and rng.random() < 0.5)
    else:
        direction = rng.choice(("forward", "backward"))
        while True:
            tokens, channels, width = size(1, 8192), size(256, 8192), size(256, 16384)
            if rng.random() < 0.6:               # channels are mostly multiples of 64, batches of anything
                channels, width = 64 * (channels // 64 | 1), 64 * (width // 64 | 1)
            if 1 << 16 <= tokens * channels * width <= 4096 * 4096 * 8192:
                break
        case = gated("", direction, tokens, channels, width, type16, rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu", "silu")),
                     bias=direction == "forward" and rng.random() < 0.5, save=direction == "forward" and rng.random() < 0.5)
    del case["name"]
    return case


def lengths(case):
    """Queries and keys of every sequence.  Causal ones have as many keys more than queries as the longest has."""
    b, q, k = case["batch"], case["q_len"], case["k_len"]
    if not case["ragged"]:
        return [q] * b, [k] * b
    part = [0.25 + 0.75 * (1 - i * 0.6180339887498949 % 1) for i in range(b)]        # 1 for the first
    qs = [max(1, int(q * p)) for p in part]
    ks = [n + k - q for n in qs] if case["causal"] else [max(1, int(k * p)) for p in part[:1] + part[:0:-1]]
    return qs, ks


def pairs(case):
    """Queries times the keys that each sees."""
    return sum(q * k - (q * (q - 1) // 2 if case["causal"] else 0) for q, k in zip(*lengths(case)))


def work(case):
    if case["op"] == "rotary":
        n = case["tokens"] * case["heads"] * case["head"]
        return {"bytes": 2 * n * BYTES[case["type"]] + 8 * case["tokens"], "flops": 3 * n}
    if case["op"] == "attention":
        (qs, ks), d, back = lengths(case), case["head"], case["direction"] == "backward"
        q, kv = sum(qs) * case["heads"] * d, sum(ks) * case["kv_heads"] * d
        count = 4 * q + 4 * kv if back else 2 * q + 2 * kv          # backward: Q, O, dO and dQ; K, V, dK and dV
        return {"bytes": 2 * count + 4 * sum(qs) * case["heads"] * (back or case["save"]),
                "flops": (10 if back else 4) * d * case["heads"] * pairs(case)}
    m, c, f = case["tokens"], case["channels"], case["width"]
    if case["direction"] == "forward":
        return {"bytes": 2 * (m * c + 2 * f * c + m * f * (3 if case["save"] else 1) + 2 * f * case["bias"]), "flops": 4 * m * c * f}
    # dY, W2, Z, X and W read, H, dZ, dX and dW written
    return {"bytes": 2 * (3 * m * c + 5 * c * f + 5 * m * f), "flops": 10 * m * c * f}


# ------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"rotary": prepare_rotary, "attention": prepare_attention, "gated": prepare_gated}[case["op"]](case, gen)


def normal(gen, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def context():
    from paper_2509_24859_amd import binding
    return binding.Context(torch.cuda.current_device())


SCALINGS = {"none": {}, "linear": {"factor": 4.0}, "ntk": {"factor": 4.0},
            "by_parts": {"factor": 8.0, "original": 8192.0, "low": 1.0, "high": 32.0}}


def prepare_rotary(case, gen):
    n, h, d, t = case["tokens"], case["heads"], case["head"], TYPES[case["type"]]
    s = {"case": case, "x": normal(gen, (n, h + case["skip"], d), t)[:, :h]}
    s["y"] = torch.empty((n, h, d), dtype=t, device="cuda")
    # positions run on from somewhere, as those of a prompt's next piece do
    first = torch.randint(0, max(1, case["far"] - n), (1,), generator=gen, device="cuda")
    s["positions"] = first + torch.arange(n, device="cuda")
    s["frequencies"], s["magnitude"] = frequencies(case)
    if own:
        s["ctx"] = context()
    return s


def frequencies(case):
    """Radians per position of each pair, in 64 bits, and what both results are multiplied by."""
    dim, how = case["turned"], SCALINGS[case["scaling"]]
    if own:
        from paper_2509_24859_amd import operators
        return operators.rotary_frequencies(context(), dim, base=BASE, scaling=case["scaling"], **how)
    base = BASE * how["factor"] ** (dim / (dim - 2)) if case["scaling"] == "ntk" else BASE
    f = [base ** (-2 * i / dim) for i in range(dim // 2)]
    if case["scaling"] == "linear":
        f = [x / how["factor"] for x in f]
    if case["scaling"] == "by_parts":       # pairs that turn often within the original context stay, others are stretched
        kept = [min(1.0, max(0.0, (how["original"] * x / (2 * math.pi) - how["low"]) / (how["high"] - how["low"]))) for x in f]
        f = [x * ((1 - g) / how["factor"] + g) for x, g in zip(f, kept)]
    magnitude = 0.1 * math.log(how["factor"]) + 1 if case["scaling"] == "by_parts" else 1.0
    return torch.tensor(f, dtype=torch.float64, device="cuda"), magnitude


def begins(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def prepare_attention(case, gen):
    (qs, ks), t = lengths(case), TYPES[case["type"]]
    h, kv, d = case["heads"], case["kv_heads"], case["head"]
    q_at, k_at = begins(qs), begins([case["k_len"]] * case["batch"] if case["padded"] else ks)
    s = {"case": case, "q_at": q_at, "k_at": k_at, "ks": ks}
    # keys that have something in common, as trained ones do: a few scores of a row stand out
    common = torch.randn((1, kv, d), generator=gen, device="cuda")
    s["q"] = normal(gen, (q_at[-1], h, d), t)
    s["k"] = (torch.randn((k_at[-1], kv, d), generator=gen, device="cuda") + 0.5 * common).to(t)
    s["v"] = normal(gen, (k_at[-1], kv, d), t)
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((h, q_at[-1]), dtype=torch.float32, device="cuda")
    # what a program keeps on the GPU of its sequences
    s["q_begin"], s["k_begin"], s["k_count"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (q_at, k_at, ks))
    if own:
        from paper_2509_24859_amd import operators
        s["ctx"] = context()
        s["workspace"] = operators.attention_workspace(s["ctx"], q_at[-1], k_at[-1], case["batch"], h, kv, d)
    if case["direction"] == "backward":
        s["do"] = normal(gen, s["q"].shape, t, 0.1)
        s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[x]) for x in ("q", "k", "v"))
        forward = dict(case, direction="forward", save=True)
        for name, x in (own_attention if own else plain_attention)(forward, s).items():
            s[name].copy_(x)
    return s


def prepare_gated(case, gen):
    m, c, f, t = case["tokens"], case["channels"], case["width"], TYPES[case["type"]]
    s = {"case": case, "w": normal(gen, (2 * f, c), t, c ** -0.5), "x": normal(gen, (m, c), t),
         "h": torch.empty((m, f), dtype=t, device="cuda")}
    s["bias"] = normal(gen, (2 * f,), t, 0.5) if case["bias"] else None
    if case["direction"] == "forward":
        s["z"] = torch.empty((m, 2 * f), dtype=t, device="cuda") if case["save"] else None
    else:
        s["w2"] = normal(gen, (c, f), t, f ** -0.5)
        s["dy"], s["z"] = normal(gen, (m, c), t, 0.1), normal(gen, (m, 2 * f), t)
        s["dz"], s["dx"], s["dw"] = torch.empty_like(s["z"]), torch.empty_like(s["x"]), torch.empty_like(s["w"])
    if own:
        from paper_2509_24859_amd import operators
        s["ctx"] = context()
        s["workspace"] = operators.gated_workspace(s["ctx"], m, f, c)
        if case["direction"] == "backward":
            s["linear"] = operators.linear_workspace(s["ctx"], m, 2 * f, c)
    return s


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if not own:
        return {"rotary": plain_rotary, "attention": plain_attention, "gated": plain_gated}[case["op"]](case, state)
    return {"rotary": own_rotary, "attention": own_attention, "gated": own_gated}[case["op"]](case, state)


def own_rotary(case, s):
    from paper_2509_24859_amd import operators
    operators.harp_rotary(s["ctx"], s["x"], s["y"], s["frequencies"], positions=s["positions"], layout=case["layout"],
                          magnitude=s["magnitude"], inverse=case["direction"] == "backward")
    return {"y": s["y"]}


def own_attention(case, s):
    from paper_2509_24859_amd import operators
    form = dict(q_begin=s["q_begin"], k_begin=s["k_begin"], k_count=s["k_count"] if case["padded"] else None,
                causal=case["causal"], workspace=s["workspace"])
    if case["direction"] == "forward":
        operators.harp_attention_forward(s["ctx"], s["q"], s["k"], s["v"], s["o"], lse=s["lse"] if case["save"] else None, **form)
        return {"o": s["o"]} | ({"lse": s["lse"]} if case["save"] else {})
    operators.harp_attention_backward(s["ctx"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"], **form)
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def own_gated(case, s):
    from paper_2509_24859_amd import operators
    if case["direction"] == "forward":
        operators.harp_gated_forward(s["ctx"], s["x"], s["w"], s["h"], bias=s["bias"], act=case["act"], z=s["z"], workspace=s["workspace"])
        return {"h": s["h"]} | ({"z": s["z"]} if case["save"] else {})
    operators.harp_gated_grad(s["ctx"], s["dy"], s["w2"], s["z"], s["dz"], h=s["h"], act=case["act"], workspace=s["workspace"])
    operators.harp_linear_grad_input(s["ctx"], s["dz"], s["w"], s["dx"], workspace=s["linear"])
    operators.harp_linear_grad_weight(s["ctx"], s["dz"], s["x"], s["dw"], workspace=s["linear"])
    return {"h": s["h"], "dz": s["dz"], "dx": s["dx"], "dw": s["dw"]}


# ------------------------------------------------------------------------------------------------- plain forms, 32 bits
def plain_rotary(case, s):
    t, r = TYPES[case["type"]], case["turned"]
    angle = s["positions"].double()[:, None] * s["frequencies"][None, :]
    if case["direction"] == "backward":
        angle = -angle
    cos, sin = ((f(angle) * s["magnitude"]).float()[:, None, :] for f in (torch.cos, torch.sin))
    x = s["x"].float()
    turned = x[..., :r]
    if case["layout"] == "half":
        a, b = turned[..., :r // 2], turned[..., r // 2:]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., r:]), -1)
    else:
        a, b = turned[..., 0::2], turned[..., 1::2]
        both = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).reshape(turned.shape)
        y = torch.cat((both, x[..., r:]), -1)
    s["y"].copy_(y.to(t))
    return {"y": s["y"]}


def plain_attention(case, s):
    """Sequence after sequence: scores [kv heads][group x queries][keys]."""
    t, h, kv, d = TYPES[case["type"]], case["heads"], case["kv_heads"], case["head"]
    group, scale, back = h // kv, case["head"] ** -0.5, case["direction"] == "backward"

    def rows(x, a, b):                       # [tokens][heads][d] -> [kv heads][group x tokens][d]
        return x[a:b].float().view(b - a, kv, group, d).permute(1, 2, 0, 3).reshape(kv, group * (b - a), d)

    def tokens(x, n):
        return x.view(kv, group, n, d).permute(2, 0, 1, 3).reshape(n, h, d).to(t)

    for b in range(case["batch"]):
        qa, qb, ka = s["q_at"][b], s["q_at"][b + 1], s["k_at"][b]
        n, m = qb - qa, s["ks"][b]
        q = rows(s["q"], qa, qb)
        k, v = (s[x][ka:ka + m].float().transpose(0, 1).contiguous() for x in ("k", "v"))        # [kv heads][keys][d]
        score = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
        if case["causal"]:
            hidden = torch.arange(m, device="cuda")[None, :] > torch.arange(n, device="cuda")[:, None] + (m - n)
            score.view(kv, group, n, m).masked_fill_(hidden, -math.inf)
        if not back:
            top = score.amax(2, keepdim=True)
            p = torch.exp(score - top)
            total = p.sum(2, keepdim=True)
            s["o"][qa:qb] = tokens(torch.matmul(p, v) / total, n)
            if case["save"]:
                s["lse"][:, qa:qb] = (top + torch.log(total)).view(h, n)
            continue
        p = torch.exp(score - s["lse"][:, qa:qb].reshape(kv, group * n, 1))
        do = rows(s["do"], qa, qb)
        delta = (do * rows(s["o"], qa, qb)).sum(2, keepdim=True)
        ds = p * (torch.matmul(do, v.transpose(1, 2).contiguous()) - delta) * scale
        s["dq"][qa:qb] = tokens(torch.matmul(ds, k), n)
        if case["padded"]:                   # keys behind the count have no gradient
            for x in ("dk", "dv"):
                s[x][ka:s["k_at"][b + 1]] = 0
        s["dk"][ka:ka + m] = torch.matmul(ds.transpose(1, 2).contiguous(), q).transpose(0, 1).to(t)
        s["dv"][ka:ka + m] = torch.matmul(p.transpose(1, 2).contiguous(), do).transpose(0, 1).to(t)
    if back:
        return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    return {"o": s["o"]} | ({"lse": s["lse"]} if case["save"] else {})


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
    if act == "silu":
        sg = 1 / (1 + torch.exp(-z))
        return sg * (1 + z * (1 - sg))
    return torch.ones_like(z)


def plain_gated(case, s):
    t, f = TYPES[case["type"]], case["width"]
    w = s["w"].float()
    if case["direction"] == "forward":
        z = s["x"].float() @ w.t()
        if case["bias"]:
            z = z + s["bias"].float()
        h = activation(z[:, :f], case["act"]) * z[:, f:]
        return {"h": h.to(t)} | ({"z": z.to(t)} if case["save"] else {})
    gate, up = s["z"][:, :f].float(), s["z"][:, f:].float()
    dh = s["dy"].float() @ s["w2"].float()
    a = activation(gate, case["act"])
    dz = torch.cat((dh * up * slope(gate, case["act"]), dh * a), 1)
    return {"h": (a * up).to(t), "dz": dz.to(t), "dx": (dz @ w).to(t), "dw": (dz.t() @ s["x"].float()).to(t)}


# ------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return {"rotary": exact_rotary, "attention": exact_attention, "gated": exact_gated}[case["op"]](case, s)


def exact_rotary(case, s):
    """As products of complex numbers."""
    r = case["turned"]
    angle = torch.outer(s["positions"].double(), s["frequencies"])
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle if case["direction"] == "forward" else -angle)[:, None, :]
    x = s["x"].double()
    y = x.clone()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = torch.complex(x[..., first], x[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return {"y": y}


def exact_attention(case, s):
    """Head after head; the backward pass by differentiation of the forward one."""
    back, group, scale = case["direction"] == "backward", case["heads"] // case["kv_heads"], case["head"] ** -0.5
    o = torch.zeros_like(s["q"], dtype=torch.float64)
    lse = torch.zeros_like(s["lse"], dtype=torch.float64)
    grads = {x: torch.zeros_like(s[x], dtype=torch.float64) for x in ("q", "k", "v")}
    for b in range(case["batch"]):
        qs = slice(s["q_at"][b], s["q_at"][b + 1])
        ks = slice(s["k_at"][b], s["k_at"][b] + s["ks"][b])
        for head in range(case["heads"]):
            kv = head // group
            q, k, v = (x.double().contiguous().requires_grad_(back) for x in (s["q"][qs, head], s["k"][ks, kv], s["v"][ks, kv]))
            score = torch.mm(q, k.t()) * scale
            if case["causal"]:
                n, m = score.shape
                seen = torch.ones((n, m), dtype=torch.bool, device="cuda").tril(m - n)
                score = score.masked_fill(~seen, -math.inf)
            total = torch.logsumexp(score, 1)
            out = torch.mm(torch.exp(score - total[:, None]), v)
            if back:
                out.backward(s["do"][qs, head].double())
                grads["q"][qs, head] = q.grad
                grads["k"][ks, kv] += k.grad
                grads["v"][ks, kv] += v.grad
            o[qs, head], lse[head, qs] = out.detach(), total.detach()
    if back:
        return {"d" + x: g for x, g in grads.items()}
    return {"o": o} | ({"lse": lse} if case["save"] else {})


def exact_gated(case, s):
    """The backward pass by differentiation of what lies behind Z, in slices of the tokens."""
    acts = {"none": lambda z: z, "relu": lambda z: z * (z > 0), "silu": lambda z: z * torch.sigmoid(z),
            "gelu": lambda z: z * 0.5 * torch.special.erfc(-z / math.sqrt(2)),
            "gelu_tanh": lambda z: z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))}
    f, w = case["width"], s["w"].double()
    x = s["x"].double()
    if case["direction"] == "forward":
        z = torch.mm(x, w.t().contiguous()) + (s["bias"].double() if case["bias"] else 0)
        h = acts[case["act"]](z[:, :f]) * z[:, f:]
        return {"h": h} | ({"z": z} if case["save"] else {})
    w2 = s["w2"].double()
    out = {"h": [], "dz": []}
    for z, dy in zip(s["z"].split(1024), s["dy"].split(1024)):
        z = z.double().requires_grad_()
        h = acts[case["act"]](z[:, :f]) * z[:, f:]
        h.backward(torch.mm(dy.double(), w2))
        out["h"].append(h.detach())
        out["dz"].append(z.grad)
    h, dz = torch.cat(out["h"]), torch.cat(out["dz"])
    return {"h": h, "dz": dz, "dx": torch.mm(dz, w), "dw": torch.mm(dz.t().contiguous(), x)}
