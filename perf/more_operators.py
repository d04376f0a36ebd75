"""Timed cases of attention over a key and value cache held in 4 bits, and of what goes with it.

Kinds of case:

  store     ``api.append_kv4`` and ``api.read_kv4``: keys and values of new tokens into pages of 4-bit codes, and the values that the cache then holds
  attend    ``api.attend_kv4``: the newest tokens of each sequence attend to its cached entries; with ``weights`` the attention that each entry got is added up
  evict     ``api.evict_kv4``: every head keeps its newest entries and of the others those with most attention, moved together into other pages
  prompt    ``api.attend_prompt``: whole prompts of several lengths, packed, with grouped heads

A vector of ``group`` channels x is stored as codes c of 4 bits, a step s and an offset m of x's type: m = min x, s = (max x - min x) / 15 in binary32, rounded
to the type, c = (x - m) / s, rounded half to even and limited to 0 .. 15.  It stands for c s + m.

With ``own`` the framework's operators run, otherwise the same results in elementary torch operations.  Inputs are drawn on the GPU: normal queries and
values, keys whose channels differ in size and have means, tables with the pages in random order, accumulated attention of long tails with ties.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------------------------------------------------- the cases

def listed():
    def store(name, B, L, ragged, at, H, D, page, group, dtype):
        return dict(name=name, kind="store", B=B, L=L, ragged=ragged, at=at, H=H, D=D, page=page, group=group, dtype=dtype)

    def attend(name, B, L, ragged, T, Hq, H, D, page, group, dtype, weights=False):
        return dict(name=name, kind="attend", B=B, L=L, ragged=ragged, T=T, Hq=Hq, H=H, D=D, page=page, group=group, dtype=dtype, weights=weights)

    def evict(name, B, L, ragged, keep, recent, H, D, page, group, dtype):
        return dict(name=name, kind="evict", B=B, L=L, ragged=ragged, keep=keep, recent=recent, H=H, D=D, page=page, group=group, dtype=dtype)

    def prompt(name, B, L, ragged, prefix, Hq, H, D, dtype, causal=True):
        return dict(name=name, kind="prompt", B=B, L=L, ragged=ragged, prefix=prefix, Hq=Hq, H=H, D=D, dtype=dtype, causal=causal)

    return [
        # one new token of each of 32 sequences that are decoded together: latency
        store("store 32 tokens", 32, 1, False, 1000, 8, 128, 64, 128, "bf16"),
        # prompts of several lengths enter the cache, fine groups
        store("store prompts", 9, 4096, True, 0, 8, 128, 16, 32, "f16"),
        # one conversation, short: the smallest call of a decoder's layer, latency
        attend("attend 1x1000", 1, 1000, False, 1, 32, 8, 128, 64, 128, "bf16"),
        # one very long document: the length has to be split
        attend("attend 1x131072", 1, 131072, False, 1, 32, 8, 128, 64, 128, "bf16"),
        # a full server: many sequences of all lengths
        attend("attend 64 ragged to 8192", 64, 8192, True, 1, 32, 8, 128, 64, 128, "bf16"),
        # nothing divides anything: four tokens a sequence to verify, seven heads a group, small pages, fine groups, attention added up
        attend("attend odd", 7, 5003, True, 4, 14, 2, 96, 16, 32, "f16", weights=True),
        # one conversation over its budget, attention added up while it was decoded
        evict("evict 1x4096", 1, 4096, False, 2048, 256, 8, 128, 64, 128, "bf16"),
        # a batch of long ones cut to a quarter
        evict("evict 16x32768", 16, 32768, True, 8191, 1000, 8, 128, 64, 64, "f16"),
        # one short prompt: latency
        prompt("prompt 1x500", 1, 500, False, 0, 32, 8, 128, "bf16"),
        # prompts of all lengths packed together
        prompt("prompt 12 ragged to 4096", 12, 4096, True, 0, 32, 8, 128, "bf16"),
        # odd heads and widths, the newer part of prompts whose beginning is there already
        prompt("prompt odd with prefix", 5, 1301, True, 777, 15, 5, 80, "f16"),
        # one long prompt: the tensor cores count
        prompt("prompt 1x16384", 1, 16384, False, 0, 32, 8, 128, "bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], uniform over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["store", "attend", "attend", "attend", "evict", "prompt", "prompt", "prompt"])
        H, per, dtype, ragged = _spread(rng, 1, 16), rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 8, 16]), rng.choice(["bf16", "f16"]), rng.random() < 0.7
        if kind == "prompt":
            case = dict(kind=kind, B=_spread(rng, 1, 64), L=_spread(rng, 1, 16384), ragged=ragged, prefix=0 if rng.random() < 0.6 else _spread(rng, 1, 8192),
                        Hq=H * per, H=H, D=rng.choice([64, 80, 96, 112, 128, 128, 128]), dtype=dtype, causal=rng.random() < 0.8)
            fits = work(case)["flops"] <= work(listed()[-1])["flops"] and case["B"] * (case["L"] + case["prefix"]) <= 1 << 16
        else:
            D = rng.choice([64, 96, 128, 128, 128])
            case = dict(kind=kind, B=_spread(rng, 1, 128), ragged=ragged, H=H, D=D, page=rng.choice([16, 32, 64, 64, 128, 256]),
                        group=rng.choice([g for g in (32, 64, 96, 128, 128) if D % g == 0]), dtype=dtype)
            if kind == "store":
                case.update(L=_spread(rng, 1, 8192), at=rng.choice([0, 0, _spread(rng, 1, 2000)]))
                fits = case["B"] * (case["L"] + case["at"]) * H * D <= 1 << 26
            elif kind == "attend":
                case.update(L=_spread(rng, 1, 131072), T=rng.choice([1, 1, 1, 2, 5, 8]), Hq=H * per, weights=rng.random() < 0.3)
                fits = case["B"] * case["L"] * H * D <= 1 << 28 and case["B"] * case["L"] * case["T"] * case["Hq"] <= 1 << 25 and case["T"] <= case["L"]
            else:
                case.update(L=_spread(rng, 1, 32768))
                case["keep"] = _spread(rng, 1, case["L"])
                case["recent"] = rng.randint(0, case["keep"])
                fits = case["B"] * case["L"] * H * D <= 1 << 28
        if fits:
            return case


def _lengths(case):
    """The sequences' lengths: those of the case, whatever the seed.  Ragged ones spread from next to nothing to L."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    least = case.get("T", 1)
    return [max(least, int(case["L"] * (rng.random() if case["ragged"] and i else 1))) for i in range(case["B"])]


# ----------------------------------------------------------------------------------------------------------------- inputs

def _keys_values(gen, n, case):
    t, H, D = TYPES[case["dtype"]], case["H"], case["D"]
    rand = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    size, mean = torch.exp(0.5 * rand(H, D)), rand(H, D)
    return (rand(n, H, D) * size + mean).to(t), rand(n, H, D).to(t)


def _table(gen, lengths, page, first=0):
    """Pages in random order for sequences of these lengths, and how many there are."""
    wide = max(1, max(-(-n // page) for n in lengths))
    order = torch.randperm(len(lengths) * wide, device="cuda", generator=gen)
    return (order.view(len(lengths), wide) + first).int(), first + len(lengths) * wide


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    kind, H, D, B, lens = case["kind"], case["H"], case["D"], case["B"], _lengths(case)
    t = TYPES[case["dtype"]]
    s = dict(case=case, lens=lens)
    if kind == "prompt":
        Hq, n = case["Hq"], sum(lens)
        fused = torch.empty(n, (Hq + 2 * H) * D, dtype=t, device="cuda")        # what one projection gives for the new tokens
        fused[:, :Hq * D] = torch.randn(n, Hq * D, device="cuda", generator=gen)
        k, v = _keys_values(gen, n, case)
        fused[:, Hq * D:(Hq + H) * D] = k.view(n, -1)
        fused[:, (Hq + H) * D:] = v.view(n, -1)
        s["q"], s["k"], s["v"] = (part.unflatten(1, (-1, D)) for part in fused.split([Hq * D, H * D, H * D], 1))
        s["starts"] = s["starts_k"] = _starts(lens)
        s["lens_k"] = [x + case["prefix"] for x in lens]
        if case["prefix"]:        # keys and values of the whole prompts stand in tensors of their own
            s["k"], s["v"] = _keys_values(gen, sum(s["lens_k"]), case)
            s["starts_k"] = _starts(s["lens_k"])
        return s
    page = case["page"]
    s["table"], pages = _table(gen, [n + case.get("at", 0) for n in lens], page)
    if kind == "evict":
        s["into"], pages = _table(gen, [min(n, case["keep"]) for n in lens], page, pages)
    if own:
        from paper_2207_08820_b200 import api
        s["cache"] = api.cache_kv4(pages, H, D, page=page, group=case["group"], dtype=t)
    else:
        s["cache"] = [dict(c=torch.zeros(pages * page, H, D, dtype=torch.uint8, device="cuda"), s=torch.zeros(pages * page, H, D // case["group"], dtype=t, device="cuda"),
                           m=torch.zeros(pages * page, H, D // case["group"], dtype=t, device="cuda")) for _ in range(2)]
    if kind == "store":
        s["k"], s["v"] = _keys_values(gen, sum(lens), case)
        s["starts"] = _starts(lens)
        s["at"] = torch.full((B,), case["at"], dtype=torch.int32, device="cuda")
        return s
    filled = s["table"].numel() * page        # every slot of the tables' pages, those behind the sequences' ends too
    step = max(page, (1 << 27) // (H * D) // page * page)
    for i in range(0, filled, step):
        n = min(step, filled - i)
        k, v = _keys_values(gen, n, case)
        if own:
            table = torch.arange(i // page, (i + n) // page, dtype=torch.int32, device="cuda").unsqueeze(0)
            api.append_kv4(k, v, s["cache"], table, torch.zeros(1, dtype=torch.int32, device="cuda"), _starts([n]))
        else:
            for to, x in zip(s["cache"], (k, v)):
                _put(to, torch.arange(i, i + n, device="cuda"), x, case)
    s["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if kind == "attend":
        s["q"] = torch.randn(B * case["T"], case["Hq"], D, device="cuda", generator=gen).to(t)
        s["starts"] = None if case["T"] == 1 else _starts([case["T"]] * B)
        s["weights"] = torch.rand(B, H, max(lens), device="cuda", generator=gen) if case["weights"] else None
    else:
        w = torch.exp(2 * torch.randn(B, H, max(lens), device="cuda", generator=gen))
        stay = [min(n, case["keep"]) for n in lens]        # what goes in and comes out again
        s["first"], s["starts"], s["total"] = torch.zeros(B, dtype=torch.int32, device="cuda"), _starts(stay), sum(stay)
        s["weights"] = torch.where(w < 0.2, torch.zeros_like(w), torch.where(w < 1, (w * 64).round() / 64, w))        # ties
    return s


# ----------------------------------------------------------------------------------------------------------------- passes

def _put(to, slots, x, case):
    """Quantises x [n, H, D] into slots: the codes by division in 64 bits, where every quotient falls on the right side of a tie."""
    n, H, D = x.shape
    for i in range(0, n, 1 << 14):
        part = x[i:i + (1 << 14)].float().view(-1, H, D // case["group"], case["group"])
        lo, hi = part.amin(-1), part.amax(-1)
        span = hi - lo
        step = (span / torch.full_like(span, 15)).to(x.dtype)
        d = step.double()
        codes = torch.round((part.double() - lo.double().unsqueeze(-1)) / torch.where(d > 0, d, torch.inf).unsqueeze(-1)).clamp(0, 15)
        at = slots[i:i + (1 << 14)]
        to["c"][at] = codes.to(torch.uint8).view(-1, H, D)
        to["s"][at], to["m"][at] = step, lo.to(x.dtype)


def _get(kept, slots, case):
    c = kept["c"][slots].float().unflatten(-1, (-1, case["group"]))
    return torch.addcmul(kept["m"][slots].float().unsqueeze(-1), c, kept["s"][slots].float().unsqueeze(-1)).flatten(-2)


def _slots(table, b, i, page):
    """Where entries i of sequence b lie."""
    return table[b].long()[i // page] * page + i % page


def _softmax(scores):
    e = torch.exp(scores - scores.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_attend(s, case):
    T, H, Hq, D, page = (case[n] for n in ("T", "H", "Hq", "D", "page"))
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    weights = s["weights"].clone() if case["weights"] else None
    for b, n in enumerate(s["lens"]):
        slots = _slots(s["table"], b, torch.arange(n, device="cuda"), page)
        k, v = (_get(part, slots, case) for part in s["cache"])        # [n, H, D]
        q = s["q"][b * T:(b + 1) * T].float().view(T, H, Hq // H, D).permute(1, 0, 2, 3).reshape(H, -1, D)
        scores = q @ k.permute(1, 2, 0) / math.sqrt(D)
        if T > 1:
            seen = torch.arange(n, device="cuda") <= torch.arange(n - T, n, device="cuda").unsqueeze(1)
            scores = scores.masked_fill(~seen.repeat_interleave(Hq // H, 0), -torch.inf)
        p = _softmax(scores)
        o = (p @ v.transpose(0, 1)).view(H, T, Hq // H, D).permute(1, 0, 2, 3)
        out[b * T:(b + 1) * T] = o.reshape(T, Hq, D).to(out.dtype)
        if weights is not None:
            weights[b, :, :n] += p.sum(1)
    return [out] + ([] if weights is None else [weights])


def _plain_evict(s, case):
    B, H, keep, recent, page = (case[n] for n in ("B", "H", "keep", "recent", "page"))
    kept = torch.full((B, H, keep), -1, dtype=torch.int32, device="cuda")
    weights, values = torch.zeros_like(s["weights"]), [[], []]
    head = torch.arange(H, device="cuda").unsqueeze(1)
    for b, n in enumerate(s["lens"]):
        stay = min(n, keep)
        old = n - min(recent, n) if n > keep else 0
        best = torch.sort(s["weights"][b, :, :old], dim=-1, descending=True, stable=True).indices[:, :stay - (n - old)]
        chosen = torch.cat([best, torch.arange(old, n, device="cuda").expand(H, -1)], 1).sort(-1).values        # [H, stay]
        kept[b, :, :stay] = chosen.int()
        weights[b, :, :stay] = s["weights"][b].gather(1, chosen)
        source, target = _slots(s["table"], b, chosen, page), _slots(s["into"], b, torch.arange(stay, device="cuda"), page)
        for part, got in zip(s["cache"], values):
            for x in part.values():
                x[target] = x[source, head].transpose(0, 1)
            got.append(_get(part, target, case).to(s["cache"][0]["s"].dtype))
    lengths = s["lengths"].clamp(max=keep)
    return [lengths, weights, kept] + [torch.cat(got) for got in values]


def _plain_prompt(s, case):
    H, Hq, D = (case[n] for n in ("H", "Hq", "D"))
    out, at, at_k = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda"), 0, 0
    for n, n_k in zip(s["lens"], s["lens_k"]):
        q = s["q"][at:at + n].float().view(n, H, Hq // H, D).permute(1, 2, 0, 3)        # [H, G, n, D]
        k, v = (s[x][at_k:at_k + n_k].float().permute(1, 0, 2).unsqueeze(1) for x in ("k", "v"))        # [H, 1, n_k, D]
        rows = max(1, min(n, (1 << 27) // (Hq * n_k)))
        for i in range(0, n, rows):
            j = min(n, i + rows)
            last = n_k - n + j if case["causal"] else n_k        # keys behind it are seen by none of these rows
            scores = q[:, :, i:j] @ k[:, :, :last].transpose(-1, -2) / math.sqrt(D)
            if case["causal"]:
                hidden = torch.arange(last, device="cuda") > torch.arange(n_k - n + i, n_k - n + j, device="cuda").unsqueeze(1)
                scores.masked_fill_(hidden, -torch.inf)
            o = _softmax(scores) @ v[:, :, :last]
            out[at + i:at + j] = o.permute(2, 0, 1, 3).reshape(j - i, Hq, D).to(out.dtype)
        at, at_k = at + n, at_k + n_k
    return out


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2207_08820_b200 import api
        if kind == "store":
            api.append_kv4(s["k"], s["v"], s["cache"], s["table"], s["at"], s["starts"])
            return api.read_kv4(s["cache"], s["table"], s["at"], s["starts"], total=s["k"].shape[0])
        if kind == "attend":
            weights = s["weights"].clone() if case["weights"] else None        # they go on adding up in a program; here every pass begins with the same
            out = api.attend_kv4(s["q"], s["cache"], s["table"], s["lengths"], s["starts"], weights=weights)
            return [out] + ([] if weights is None else [weights])
        if kind == "evict":
            lengths, weights, kept = api.evict_kv4(s["cache"], s["table"], s["lengths"], s["weights"], case["keep"], recent=case["recent"], into=s["into"])
            return [lengths, weights, kept, *api.read_kv4(s["cache"], s["into"], s["first"], s["starts"], total=s["total"])]
        return api.attend_prompt(s["q"], s["k"], s["v"], s["starts"], s["starts_k"], causal=case["causal"])
    if kind == "store":
        i = torch.arange(s["k"].shape[0], device="cuda")
        b = torch.bucketize(i, s["starts"].long()[1:], right=True)
        i = i - s["starts"].long()[b] + s["at"].long()[b]
        slots = s["table"].long()[b, i // case["page"]] * case["page"] + i % case["page"]
        for to, x in zip(s["cache"], (s["k"], s["v"])):
            _put(to, slots, x, case)
        return tuple(_get(part, slots, case).to(s["k"].dtype) for part in s["cache"])
    if kind == "attend":
        return _plain_attend(s, case)
    if kind == "evict":
        return _plain_evict(s, case)
    return _plain_prompt(s, case)


# ------------------------------------------------------------------------------------------------------------ what it costs

def work(case):
    lens, H, D = _lengths(case), case["H"], case["D"]
    if case["kind"] == "prompt":
        seen = sum(n * case["prefix"] + (n * (n + 1) // 2 if case["causal"] else n * n) for n in lens)
        return dict(bytes=2 * D * sum(2 * case["Hq"] * n + 2 * H * (n + case["prefix"]) for n in lens), flops=4 * D * case["Hq"] * seen)
    entry = H * (D + 8 * (D // case["group"]))        # codes, steps and offsets of a token's keys and values
    if case["kind"] == "store":
        return dict(bytes=sum(lens) * (2 * entry + 8 * H * D), flops=0)
    if case["kind"] == "attend":
        rows = case["T"] * case["Hq"]
        return dict(bytes=sum(lens) * (entry + (8 * H if case["weights"] else 0)) + 4 * case["B"] * rows * D, flops=4 * D * rows * sum(lens))
    stay = sum(min(n, case["keep"]) for n in lens)
    return dict(bytes=sum(lens) * 4 * H + stay * (3 * entry + 8 * H + 4 * H * D), flops=0)


# ------------------------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_values(x, group, dtype):
    """The values that codes, steps and offsets of x [..., D] stand for."""
    parts = []
    for c in range(0, x.shape[-1], group):
        u = x[..., c:c + group].double()
        lo, hi = u.min(-1, keepdim=True).values, u.max(-1, keepdim=True).values
        step = ((hi - lo).float() / torch.tensor(15.0, device=x.device).expand(lo.shape)).to(dtype).double()        # its roundings are the format's
        q = torch.nan_to_num((u - lo) / step, nan=0.0, posinf=0.0).round().clamp(0, 15)
        parts.append(q * step + lo)
    return torch.cat(parts, -1)


def _exact_rows(q, k, v, seen, D):
    """One head: rows q [r, D], entries k, v [n, D], which entry each row sees [r, n]."""
    a = (q @ k.T) * D ** -0.5
    a = torch.where(seen, a, torch.full_like(a, -math.inf))
    p = torch.exp(a - a.max(1, keepdim=True).values)
    p = p / p.sum(1, keepdim=True)
    return p @ v, p


def exact(case, seed):
    global own
    kind, H, D = case["kind"], case["H"], case["D"]
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    t = TYPES[case["dtype"]]
    if kind == "store":
        return tuple(_exact_values(s[x], case["group"], t) for x in ("k", "v"))
    if kind == "prompt":
        out, group, at, at_k = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), case["Hq"] // H, 0, 0
        for n, n_k in zip(s["lens"], s["lens_k"]):
            for h in range(case["Hq"]):
                k, v = s["k"][at_k:at_k + n_k, h // group].double(), s["v"][at_k:at_k + n_k, h // group].double()
                for i in range(0, n, 4096):
                    j = min(n, i + 4096)
                    key, row = torch.arange(n_k, device="cuda"), torch.arange(i, j, device="cuda").unsqueeze(1)
                    seen = key - (n_k - n) <= row if case["causal"] else key >= 0 * row
                    out[at + i:at + j, h] = _exact_rows(s["q"][at + i:at + j, h].double(), k, v, seen, D)[0]
            at, at_k = at + n, at_k + n_k
        return out

    def held(part, where, h):        # entries of one head, out of the codes that prepare made by the formula
        c, step, m = (part[x][where, h].double() for x in ("c", "s", "m"))
        which = torch.arange(D, device="cuda") // case["group"]
        return c * step[:, which] + m[:, which]

    def place(table, b, i):
        return table[b].long().gather(0, torch.div(i, case["page"], rounding_mode="floor")) * case["page"] + torch.remainder(i, case["page"])

    if kind == "attend":
        T, group = case["T"], case["Hq"] // H
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        weights = s["weights"].double() if case["weights"] else None
        for b, n in enumerate(s["lens"]):
            entry = torch.arange(n, device="cuda")
            where = place(s["table"], b, entry)
            seen = entry <= (n - T + torch.arange(T, device="cuda")).unsqueeze(1)
            for h in range(H):
                k, v = (held(part, where, h) for part in s["cache"])
                for g in range(h * group, (h + 1) * group):
                    out[b * T:(b + 1) * T, g], p = _exact_rows(s["q"][b * T:(b + 1) * T, g].double(), k, v, seen, D)
                    if weights is not None:
                        weights[b, h, :n] += p.sum(0)
        return [out] + ([] if weights is None else [weights])
    keep, recent = case["keep"], case["recent"]
    weights, values = torch.zeros(s["weights"].shape, dtype=torch.float64, device="cuda"), ([], [])
    for b, n in enumerate(s["lens"]):
        rows = ([], [])
        for h in range(H):
            w = s["weights"][b, h, :n].double()
            if n > keep:
                rank = torch.argsort(torch.cat([-w[:n - recent], torch.full((recent,), -math.inf, device="cuda", dtype=torch.float64)]), stable=True)
                chosen = rank[:keep].sort().values
            else:
                chosen = torch.arange(n, device="cuda")
            weights[b, h, :len(chosen)] = w[chosen]
            for part, to in zip(s["cache"], rows):
                to.append(held(part, place(s["table"], b, chosen), h))
        for to, got in zip(rows, values):
            got.append(torch.stack(to, 1))
    return [None, weights, None] + [torch.cat(got) for got in values]
