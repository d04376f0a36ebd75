"""The operators on grouped 4-bit weights from their definitions, in 64 bits on the CPU, with the bounds that their roundings allow."""
import numpy as np
import torch

F32_STEP = 2.0 ** -22       # one addition of the tensor cores: 32-bit sums whose addends may be cut off instead of rounded, four times the half step of a float


def round_half_even(v):
    return np.rint(v)


def quantise(w, group, zeros, dtype):
    """(codes, scales, zero points) of float weights [O, K]; scales as the type's values in float64."""
    w = w.double().numpy()
    O, K = w.shape
    G = -(-K // group)
    codes, scales, zps = np.zeros((O, K), np.int8), np.zeros((O, G)), np.zeros((O, G), np.int8)
    top = torch.finfo(dtype).max
    f32, narrow = np.float32, lambda v: torch.from_numpy(np.ascontiguousarray(v)).to(dtype).double().numpy()
    with np.errstate(all="ignore"):
        for g in range(G):
            part = w[:, g * group:(g + 1) * group]
            known = np.where(np.isnan(part), 0.0, part)
            lo, hi = np.minimum(known.min(1), 0), np.maximum(known.max(1), 0)
            if zeros:
                wide = (f32(hi) - f32(lo)).astype(f32) / f32(15)
            else:
                wide = f32(np.maximum(hi, -lo)) / f32(7)
            s = narrow(np.minimum(wide.astype(f32), f32(top)))
            scales[:, g] = s
            safe = np.where(s > 0, s, 1.0)
            z = np.where(s > 0, np.clip(round_half_even(-lo / safe), 0, 15), 0) if zeros else np.zeros(O)
            zps[:, g] = z
            q = round_half_even(part / safe[:, None]) + z[:, None]
            low, high = (0, 15) if zeros else (-8, 7)
            q = np.where(np.isnan(q), low, np.clip(q, low, high))
            codes[:, g * group:(g + 1) * group] = np.where(s[:, None] > 0, q, z[:, None])
    return codes, scales, zps


def matrix(codes, scales, zeros, group):
    """The weights that codes, scales and zero points stand for."""
    K = codes.shape[-1]
    at = torch.arange(K) // group
    q = codes.double()
    if zeros is not None:
        q = q - zeros.double()[..., at]
    return q * scales.double()[..., at]


def half_step(y, dtype):
    """The last rounding: half a step of the value, or of the smallest normal one."""
    f = torch.finfo(dtype)
    return f.eps / 2 * y.abs().clamp(min=f.tiny)


def sum_error(K, size):
    """Bound on K products' 32-bit sum in MMAs of 16, warps' parts and scaled groups, `size` the sum of the products' magnitudes."""
    return (K / 16 + 3 * (K / 32 + 1) + 16) * F32_STEP * size


def gemm(x, w, bias, dtype):
    """(y, how far off it may be) of x [M, K] and weights [O, K] in float64."""
    x = x.double()
    y, size = x @ w.T, x.abs() @ w.abs().T
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return y, half_step(y, dtype) + sum_error(x.shape[1], size) * (1 + torch.finfo(dtype).eps)


def moe(x, router, gate, up, down, top_k, renormalise, dtype):
    """(y, its bound, experts, weights): weights of the experts [E, I, H], [E, I, H], [E, H, I] in float64."""
    x = x.double()
    logits = x @ router.double().T
    experts = torch.sort(-logits, dim=-1, stable=True).indices[:, :top_k]
    p = torch.exp(logits - logits.max(-1, keepdim=True).values)
    chosen = p.gather(1, experts)
    weights = chosen / (chosen if renormalise else p).sum(-1, keepdim=True)
    y, far = torch.zeros_like(x), torch.zeros_like(x)
    H, I = x.shape[1], gate.shape[1]
    for t in range(x.shape[0]):
        for j, e in enumerate(experts[t].tolist()):
            g, u = gate[e] @ x[t], up[e] @ x[t]
            dg, du = (sum_error(H, w[e].abs() @ x[t].abs()) for w in (gate, up))
            silu = g * torch.sigmoid(g)
            h = silu * u * weights[t, j]
            # silu is at most 1.1 steep; expf, the quotient and the weight are a few steps of a float off; hi + lo keep 2^-9 * 2^-9 of a value
            dh = (1.1 * dg * (u.abs() + du) + silu.abs() * du) * weights[t, j] + h.abs() * (2.0 ** -19 + 2.0 ** -17)
            y[t] += down[e] @ h
            far[t] += down[e].abs() @ dh + sum_error(2 * I, down[e].abs() @ h.abs())
    return y, far * (1 + torch.finfo(dtype).eps) + half_step(y, dtype), experts, weights
