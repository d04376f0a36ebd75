"""Timed cases of the operators on grouped 4-bit weights: the quantiser, the product with 16-bit activations, the mixture-of-experts layer.

Kinds of case:

  quantise    ``api.quantise_w4``: float weights [O, K] to codes, one scale (and zero point) per group of a row
  linear      ``api.gemm_w4``: y = x W^T + bias with W[o, k] = scale[o, k // group] * (code[o, k] - zero[o, k // group])
  moe         ``api.moe_w4``: router, the best experts of each token, gated experts of such weights, weighted sum

With ``own`` the framework's operators run, otherwise the same results in elementary torch operations.  Inputs are drawn on the GPU: normal
activations, codes of normal weights, scales that spread by a factor of three.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------------------- the cases

def listed():
    def linear(name, M, O, K, group, dtype, zeros, bias):
        return dict(name=name, kind="linear", M=M, O=O, K=K, group=group, dtype=dtype, zeros=zeros, bias=bias)

    def moe(name, T, E, top_k, H, I, group, dtype, zeros, renormalise):
        return dict(name=name, kind="moe", T=T, E=E, top_k=top_k, H=H, I=I, group=group, dtype=dtype, zeros=zeros, renormalise=renormalise)

    def quantise(name, O, K, group, source, dtype, zeros):
        return dict(name=name, kind="quantise", O=O, K=K, group=group, source=source, dtype=dtype, zeros=zeros)

    return [
        # one token through a square projection: the smallest call, latency
        linear("linear 1x4096x4096", 1, 4096, 4096, 128, "bf16", False, False),
        # one token through the widest layer: the weights come from HBM in every pass
        linear("linear 1x24576x8192", 1, 24576, 8192, 128, "bf16", False, False),
        # eight sequences decoded together, zero points, finer groups
        linear("linear 8x16384x4096 zeros", 8, 16384, 4096, 64, "f16", True, True),
        # nothing divides anything: odd tokens, outputs and reduction, the finest groups
        linear("linear 33x1383x4611 odd", 33, 1383, 4611, 32, "bf16", True, True),
        # a short prompt: weights and arithmetic cost alike
        linear("linear 200x4096x4096", 200, 4096, 4096, 128, "f16", False, True),
        # a long prompt: the tensor cores count
        linear("linear 4096x16384x4096", 4096, 16384, 4096, 128, "bf16", False, False),
        # one token, many small experts
        moe("moe 1 of 64 experts", 1, 64, 8, 2048, 1024, 128, "bf16", False, True),
        # a few sequences, few large experts
        moe("moe 8 of 16 experts", 8, 16, 2, 4096, 8192, 128, "bf16", False, True),
        # odd widths and tokens, zero points, weights that are not renormalised
        moe("moe 37 of 60 experts odd", 37, 60, 4, 2001, 1390, 32, "f16", True, False),
        # the largest batch of tokens that counts as a few: nearly all experts are read
        moe("moe 64 of 128 experts", 64, 128, 8, 2048, 768, 128, "bf16", False, True),
        # weights quantised when a model is loaded: one projection of a float32 checkpoint, and the widest layer with zero points
        quantise("quantise 4096x4096 f32", 4096, 4096, 128, "f32", "bf16", False),
        quantise("quantise 24576x8192 zeros", 24576, 8192, 64, "bf16", "bf16", True),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], uniform over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["linear", "linear", "linear", "moe", "moe", "quantise"])
        size = lambda lo, hi: _spread(rng, lo, hi) if rng.random() < 0.4 else 64 * _spread(rng, max(1, lo // 64), hi // 64)  # noqa: E731
        case = dict(kind=kind, group=rng.choice([32, 64, 128, 128, 256]), dtype=rng.choice(["bf16", "f16"]), zeros=rng.random() < 0.4)
        if kind == "linear":
            case.update(M=_spread(rng, 1, 4096), O=size(64, 24576), K=size(64, 8192), bias=rng.random() < 0.5)
            fits = case["M"] * case["O"] * case["K"] <= 4096 * 16384 * 4096 and case["O"] * case["K"] >= 1 << 18
        elif kind == "moe":
            case.update(T=_spread(rng, 1, 64), E=_spread(rng, 4, 128), H=size(256, 4096), I=size(128, 8192), renormalise=rng.random() < 0.5)
            case["top_k"] = rng.randint(1, min(8, case["E"]))
            fits = case["E"] * case["H"] * case["I"] <= 16 * 4096 * 8192
        else:
            case.update(O=size(64, 24576), K=size(64, 8192), source=rng.choice(["f32", "bf16", "f16"]))
            fits = True
        if fits:
            return case


# ----------------------------------------------------------------------------------------------------------------- inputs

def _weights(gen, lead, O, K, case):
    """Codes, scales and zero points of weights of about 1 / sqrt(K)."""
    G, t = -(-K // case["group"]), TYPES[case["dtype"]]
    codes = torch.empty(*lead, O, K, dtype=torch.int8, device="cuda")
    for part in codes.view(-1, K).split(1 << 13):        # a part at a time: the normal draws are wider than the codes
        part.copy_(torch.randn(part.shape, device="cuda", dtype=torch.float16, generator=gen).mul_(2.8).round_().clamp_(-8, 7))
    scales = ((torch.rand(*lead, O, G, device="cuda", generator=gen) + 0.5) * (0.36 / math.sqrt(K))).to(t)
    zeros = None
    if case["zeros"]:
        zeros = torch.randint(6, 11, (*lead, O, G), device="cuda", dtype=torch.int8, generator=gen)
        codes += 8
    return codes, scales, zeros


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    s = dict(case=case)
    if case["kind"] == "quantise":
        s["w"] = (torch.randn(case["O"], case["K"], device="cuda", generator=gen) / math.sqrt(case["K"])).to(TYPES[case["source"]])
        return s
    t = TYPES[case["dtype"]]
    if case["kind"] == "linear":
        s["x"] = torch.randn(case["M"], case["K"], device="cuda", generator=gen).to(t)
        s["bias"] = torch.randn(case["O"], device="cuda", generator=gen).to(t) if case["bias"] else None
        s["w"] = _weights(gen, (), case["O"], case["K"], case)
    else:
        T, E, H, I = case["T"], case["E"], case["H"], case["I"]
        s["x"] = torch.randn(T, H, device="cuda", generator=gen).to(t)
        s["router"] = (torch.randn(E, H, device="cuda", generator=gen) / math.sqrt(H)).to(t)
        s["gate"], s["up"], s["down"] = (_weights(gen, (E,), o, k, case) for o, k in ((I, H), (I, H), (H, I)))
    if own:
        from paper_2207_08820_b200 import api
        for name in ("w", "gate", "up", "down"):
            if name in s:
                s[name] = api.prepare_w4(*s[name], group=case["group"])
    return s


# ----------------------------------------------------------------------------------------------------------------- passes

def _matrix(w, group, K, to=torch.float32):
    codes, scales, zeros = w
    centred = codes.to(to)
    if zeros is not None:
        centred = centred - zeros.to(to).repeat_interleave(group, -1)[..., :K]
    return centred * scales.to(to).repeat_interleave(group, -1)[..., :K]


def _plain_quantise(w, case):
    """Codes by division in 64 bits, where every quotient falls on the right side of a tie; scales by one division in 32 bits."""
    O, K, group, t = case["O"], case["K"], case["group"], TYPES[case["dtype"]]
    G = -(-K // group)
    v = torch.nn.functional.pad(w.float(), (0, G * group - K)).view(O, G, group)
    if case["zeros"]:
        lo, hi = v.amin(-1).clamp(max=0), v.amax(-1).clamp(min=0)
        span = hi - lo
        scales = span / torch.full_like(span, 15)
    else:
        span = v.abs().amax(-1)
        scales = span / torch.full_like(span, 7)
    scales = scales.clamp(max=torch.finfo(t).max).to(t)
    step = scales.double()
    step = torch.where(step > 0, step, torch.inf)
    codes = torch.round(v.double() / step.unsqueeze(-1))
    zeros = None
    if case["zeros"]:
        zeros = torch.round(-lo.double() / step).clamp(0, 15)
        codes = (codes + zeros.unsqueeze(-1)).clamp(0, 15)
        zeros = zeros.to(torch.int8)
    else:
        codes = codes.clamp(-8, 7)
    codes = codes.to(torch.int8).view(O, G * group)[:, :K].contiguous()
    return [codes, scales] + ([] if zeros is None else [zeros])


def _choose(logits, case):
    """The best experts of each token, ties to the lowest index, and their weights."""
    p = torch.softmax(logits, -1)
    experts = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :case["top_k"]]
    weights = p.gather(-1, experts)
    if case["renormalise"]:
        weights = weights / weights.sum(-1, keepdim=True)
    return experts, weights


def _plain_moe(s, case):
    T, E, k, H, I, g = (case[n] for n in ("T", "E", "top_k", "H", "I", "group"))
    x = s["x"].float()
    # the order of the experts is decided in 64 bits
    experts, weights = _choose(s["x"].double() @ s["router"].double().T, case)
    if T * k < E:        # each choice with its own expert's weights
        at = experts.reshape(-1)
        pick = lambda w: [None if p is None else p[at] for p in w]  # noqa: E731
        xs = x.repeat_interleave(k, 0).unsqueeze(-1)
        gate, up = (_matrix(pick(s[n]), g, H) @ xs for n in ("gate", "up"))
        hidden = gate * torch.sigmoid(gate) * up
        y = (_matrix(pick(s["down"]), g, I) @ hidden).view(T, k, H)
        y = (y * weights.float().unsqueeze(-1)).sum(1)
    else:                # all experts on all tokens, weighted by what was chosen
        gate, up = (x @ _matrix(s[n], g, H).transpose(1, 2) for n in ("gate", "up"))
        share = torch.zeros(T, E, device="cuda").scatter_(1, experts, weights.float())
        hidden = gate * torch.sigmoid(gate) * up * share.T.unsqueeze(-1)
        y = torch.bmm(hidden, _matrix(s["down"], g, I).transpose(1, 2)).sum(0)
    return y.to(s["x"].dtype), experts.int(), weights.float()


def run(s):
    case = s["case"]
    if own:
        from paper_2207_08820_b200 import api
        if case["kind"] == "quantise":
            return [v for v in api.quantise_w4(s["w"], case["group"], zeros=case["zeros"], dtype=TYPES[case["dtype"]]) if v is not None]
        if case["kind"] == "linear":
            return api.gemm_w4(s["x"], s["w"], s["bias"])
        return api.moe_w4(s["x"], s["router"], s["gate"], s["up"], s["down"], case["top_k"], renormalise=case["renormalise"])
    if case["kind"] == "quantise":
        return _plain_quantise(s["w"], case)
    if case["kind"] == "linear":
        y = s["x"].float() @ _matrix(s["w"], case["group"], case["K"]).T
        if s["bias"] is not None:
            y = y + s["bias"].float()
        return y.to(s["x"].dtype)
    return _plain_moe(s, case)


# ------------------------------------------------------------------------------------------------------------ what it costs

def _weight_bytes(O, K, case):
    return O * K / 2 + O * -(-K // case["group"]) * (2.5 if case["zeros"] else 2)


def work(case):
    if case["kind"] == "quantise":
        O, K = case["O"], case["K"]
        return dict(bytes=O * K * ((4 if case["source"] == "f32" else 2) + 1) + O * -(-K // case["group"]) * (3 if case["zeros"] else 2), flops=0)
    if case["kind"] == "linear":
        M, O, K = case["M"], case["O"], case["K"]
        return dict(bytes=_weight_bytes(O, K, case) + 2 * M * (O + K) + (2 * O if case["bias"] else 0), flops=2 * M * O * K)
    T, E, k, H, I = (case[n] for n in ("T", "E", "top_k", "H", "I"))
    read = E * (1 - (1 - k / E) ** T)        # experts that some token chose, on average
    return dict(bytes=read * (2 * _weight_bytes(I, H, case) + _weight_bytes(H, I, case)) + 2 * E * H + 4 * T * H + 8 * T * k,
                flops=2 * T * (3 * k * H * I + E * H))


# ------------------------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_rows(w, group, rows=slice(None)):
    """Rows of the weights that codes, scales and zero points stand for."""
    codes, scales, zeros = w
    q, s = codes[rows].double(), scales[rows].double()
    which = torch.arange(q.shape[-1], device=q.device) // group
    if zeros is not None:
        q = q - zeros[rows].double()[..., which]
    return q * s[..., which]


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "quantise":
        w, O, K, group = s["w"].double(), case["O"], case["K"], case["group"]
        scales = torch.empty(O, -(-K // group), dtype=torch.float64, device="cuda")
        for g in range(scales.shape[1]):
            part = w[:, g * group:(g + 1) * group]
            if case["zeros"]:
                scales[:, g] = (part.max(1).values.clamp(min=0) - part.min(1).values.clamp(max=0)) / 15
            else:
                scales[:, g] = part.abs().max(1).values / 7
        return [None, scales] + ([None] if case["zeros"] else [])
    x, group = s["x"].double(), case["group"]
    if case["kind"] == "linear":
        y = torch.empty(case["M"], case["O"], dtype=torch.float64, device="cuda")
        for o in range(0, case["O"], 4096):
            y[:, o:o + 4096] = x @ _exact_rows(s["w"], group, slice(o, o + 4096)).T
        return y if s["bias"] is None else y + s["bias"].double()
    logits = x @ s["router"].double().T
    best = torch.sort(-logits, dim=-1, stable=True).indices[:, :case["top_k"]]
    e = torch.exp(logits - logits.max(-1, keepdim=True).values)
    chosen = e.gather(1, best)
    weights = chosen / (chosen.sum(1, keepdim=True) if case["renormalise"] else e.sum(1, keepdim=True))
    y = torch.zeros_like(x)
    for expert in best.unique().tolist():
        token, place = (best == expert).nonzero(as_tuple=True)
        u = x[token]
        gate, up = u @ _exact_rows(s["gate"], group, expert).T, u @ _exact_rows(s["up"], group, expert).T
        hidden = gate / (1 + torch.exp(-gate)) * up
        y.index_add_(0, token, (hidden @ _exact_rows(s["down"], group, expert).T) * weights[token, place].unsqueeze(1))
    return y, None, weights
