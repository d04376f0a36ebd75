"""Attention over a cache of 4-bit keys and values by its definition, in 64 bits on the CPU, and bounds that count each rounding of the kernels."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # a rounding, relative to the value


def quantise(x, group):
    """x [..., D] of 16 bits: (codes, steps, offsets) in 64 bits, groups on an axis of their own."""
    v = x.float().unflatten(-1, (-1, group))
    lo, hi = v.amin(-1), v.amax(-1)
    span = hi - lo
    step = (span / torch.full_like(span, 15)).to(x.dtype).double()
    c = torch.round((v.double() - lo.double().unsqueeze(-1)) / torch.where(step > 0, step, torch.inf).unsqueeze(-1)).clamp(0, 15)
    bad = ~torch.isfinite(v).all(-1) | ~torch.isfinite(span)
    return torch.where(bad.unsqueeze(-1), 0.0, c), torch.where(bad, 0.0, step), torch.where(bad, math.nan, lo.double())


def values(x, group):
    """What the cache holds of x, in 64 bits."""
    c, s, m = quantise(x, group)
    return (c * s.unsqueeze(-1) + m.unsqueeze(-1)).flatten(-2)


def read(x, group):
    """What read_kv4 gives for x: one rounding to binary32, one to the type."""
    return values(x, group).float().to(x.dtype)


def parts(x, group):
    """Bounds of what the kernels add up for a value: c s + |m|, and the steps."""
    c, s, m = quantise(x, group)
    return (c * s.unsqueeze(-1) + m.abs().unsqueeze(-1)).flatten(-2), s


def attend(q, k, v, group, scale=None):
    """q [t, Hq, D], a sequence's entries k, v [n, H, D] as they were stored (16 bits).  Returns out [t, Hq, D] and what each entry gets [H, n] in 64 bits, and how
    far off they may be."""
    (t, Hq, D), (n, H) = q.shape, k.shape[:2]
    scale = D ** -0.5 if scale is None else scale
    per, half = Hq // H, HALF[q.dtype]
    out, far = torch.zeros(t, Hq, D, dtype=torch.float64), torch.zeros(t, Hq, D, dtype=torch.float64)
    got, got_far = torch.zeros(H, n, dtype=torch.float64), torch.zeros(H, n, dtype=torch.float64)
    if n == 0 or t == 0:
        return out, far, got, got_far
    kk, vv = values(k, group), values(v, group)
    (kp, _), (vp, vs) = parts(k, group), parts(v, group)
    seen = torch.arange(n) <= (n - t + torch.arange(t)).unsqueeze(1)
    for j in range(Hq):
        h = j // per
        a = scale * (q[:, j].double() @ kk[:, h].T)
        a = torch.where(seen, a, -math.inf)
        top = a.amax(1, keepdim=True)
        e = torch.where(seen, torch.exp(a - torch.where(top > -math.inf, top, 0)), 0.0)
        total = e.sum(1, keepdim=True)
        p = torch.where(total > 0, e / total, 0.0)
        out[:, j] = p @ vv[:, h]
        # a score: D / 16 + a few additions in 32 bits (the tensor core's may lose a unit of the last place of the largest term each), of terms q c s and q m;
        # then three roundings of the product with the scale and the distance from the maximum, and the exponential's 2^-22
        # (the queries brought to fp16 lose 2^-38 of the largest one)
        size = q[:, j].double().abs() @ kp[:, h].T
        off = scale * size * (D / 16 + 8) * 2.0 ** -23 + 2.0 ** -38 * scale * q[:, j].double().abs().amax(1, keepdim=True) * kp[:, h].sum(1)
        off = off + 3 * 2.0 ** -24 * (scale * size).amax(1, keepdim=True) * 2
        rel = torch.where(seen, torch.expm1((off.amax(1, keepdim=True) + off).clamp(max=50)) + 2.0 ** -20, 0.0)
        # outputs: n sums in 32 bits, weights in two fp16 terms (2^-22 of them, 2^-25 of the largest step where they are small, times codes up to 15), or for bf16 in one (2^-11)
        sums = (n / 16 + 16) * 2.0 ** -24
        weight = p * (2 * rel + 2 * (p * rel).sum(1, keepdim=True) + sums + (2.0 ** -22 if q.dtype == torch.float16 else 2.0 ** -11))
        floor = torch.where(total > 0, n * 15 * 2.0 ** -25 * 2 * vs[:, h].max() / total.clamp(min=1e-300), 0.0)
        far[:, j] = weight @ vp[:, h] + floor
        far[:, j] += half * (out[:, j].abs() + far[:, j]) + torch.finfo(q.dtype).smallest_normal * torch.finfo(q.dtype).eps
        got[h] += p.sum(0)
        got_far[h] += (p * (2 * rel + 2 * (p * rel).sum(1, keepdim=True) + sums)).sum(0)
    return out, far, got, got_far + 2.0 ** -24 * (t * per + 2) * got


def evict(weights, n, keep, recent):
    """Indices that stay, of one head of a sequence of n entries."""
    if n <= keep:
        return torch.arange(n)
    old = n - recent
    w = weights[:old].double()
    w = torch.where(torch.isnan(w), math.inf, w)
    first = torch.isnan(weights[:old])
    order = sorted(range(old), key=lambda i: (not bool(first[i]), -float(w[i]), i))[:keep - recent]
    return torch.tensor(sorted(order) + list(range(old, n)), dtype=torch.long)
