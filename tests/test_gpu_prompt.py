"""Attention of whole prompts on the GPU against its definition in 64 bits.  Bounds count the roundings: scores in 32 bits, weights rounded to the type, the last one."""
import math

import pytest
import torch

from kv4_reference import HALF
from paper_2207_08820_b200 import api
from paper_2207_08820_b200._lib import BitserialError

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
GUARD = 77.0


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def starts_of(counts, first=0):
    return ints([first] + (torch.tensor(counts, dtype=torch.long).cumsum(0) + first).tolist())


def reference(q, k, v, causal=True, scale=None):
    """One sequence, on the GPU in 64 bits: q [n, Hq, D], k and v [m, H, D].  Returns out and how far off it may be."""
    (n, Hq, D), (m, H) = q.shape, k.shape[:2]
    scale = D ** -0.5 if scale is None else scale
    out, far = torch.zeros(n, Hq, D, dtype=torch.float64, device="cuda"), torch.zeros(n, Hq, D, dtype=torch.float64, device="cuda")
    if n == 0 or m == 0:
        return out, far
    seen = torch.arange(m, device="cuda") <= (m - n + torch.arange(n, device="cuda")).unsqueeze(1) if causal else torch.ones(n, m, dtype=torch.bool, device="cuda")
    u = HALF[q.dtype]
    for h in range(Hq):
        qd, kd, vd = q[:, h].double(), k[:, h // (Hq // H)].double(), v[:, h // (Hq // H)].double()
        a = torch.where(seen, scale * (qd @ kd.T), -math.inf)
        top = a.amax(1, keepdim=True)
        e = torch.where(seen, torch.exp(a - torch.where(top > -math.inf, top, 0)), 0.0)
        total = e.sum(1, keepdim=True)
        p = torch.where(total > 0, e / total, 0.0)
        out[:, h] = p @ vd
        # a score: D / 16 additions in the tensor core and three roundings; the exponential 2^-21; the weight's own rounding, and 2^-25 of the largest weight where fp16
        # holds it with fewer bits; sums of up to m / 16 products in the tensor core
        size = scale * (qd.abs() @ kd.abs().T)
        off = size * (D / 16 + 4) * 2.0 ** -23 + 4 * 2.0 ** -24 * size.amax(1, keepdim=True)
        rel = torch.where(seen, torch.expm1((off + off.amax(1, keepdim=True)).clamp(max=50)) + 2.0 ** -20, 0.0)
        bound = p * (rel + (p * rel).sum(1, keepdim=True) + u + (m / 16 + 8) * 2.0 ** -23)
        floor = torch.where(total > 0, 2.0 ** -25 / total.clamp(min=1e-300), 0.0) * vd.abs().sum(0) if q.dtype == F16 else 0.0
        far[:, h] = bound @ vd.abs() + floor
        far[:, h] += u * (out[:, h].abs() + far[:, h]) + torch.finfo(q.dtype).smallest_normal * torch.finfo(q.dtype).eps
    return out, far


def check(counts, counts_k, Hq, H, D, dtype, causal=True, scale=None, seed=1, size=1.0):
    """Packed sequences out of views of wider tensors, NaN between and behind them; guard values around the output."""
    gen = torch.Generator("cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    T, Tk = sum(counts), sum(counts_k)
    wide_q = torch.full((T + 5, Hq + 2 * H, D), math.nan, dtype=dtype, device="cuda")
    wide_k, wide_v = (torch.full((Tk + 200, H + 1, D), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    q, k, v = wide_q[:, :Hq], wide_k[:, 1:], wide_v[:, :H]
    q[2:T + 2], k[3:Tk + 3], v[3:Tk + 3] = (rand(T, Hq, D) * size).to(dtype), rand(Tk, H, D).to(dtype), (rand(Tk, H, D) + 0.5).to(dtype)
    room = torch.full((T + 7, Hq, D), GUARD, dtype=dtype, device="cuda")
    out = api.attend_prompt(q, k, v, starts_of(counts, 2), starts_of(counts_k, 3), causal=causal, scale=scale, out=room[1:T + 6])
    api.bs_check_status()
    assert (room[:3] == GUARD).all() and (room[T + 3:] == GUARD).all()
    i, j = 2, 3
    for n, m in zip(counts, counts_k):
        want, far = reference(q[i:i + n], k[j:j + m], v[j:j + m], causal, scale)
        off = (out[i:i + n].double() - want).abs()
        assert (off <= far).all(), (n, m, (off / far).max())
        i, j = i + n, j + m


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("D", [8, 40, 64, 72, 80, 96, 112, 128])
def test_widths(D, dtype):
    check([1, 130, 300], [1, 130, 300], 4, 2, D, dtype)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 700])
def test_lengths(n, causal):
    check([n], [n], 2, 1, 128, BF16, causal)
    check([n, 3, n], [n, 3, n], 8, 2, 64, F16, causal)


@pytest.mark.parametrize("Hq,H", [(1, 1), (3, 3), (6, 2), (5, 1), (7, 1), (12, 1), (16, 2), (64, 1), (100, 1), (128, 1)])
def test_heads(Hq, H):
    check([70, 1, 290], [70, 1, 290], Hq, H, 128, BF16)


@pytest.mark.parametrize("causal", [True, False])
def test_queries_and_keys_of_other_numbers(causal):
    """Prompts whose beginning is there already, and more rows than keys: the first rows of these see nothing."""
    check([5, 100, 300, 1, 260, 40], [500, 129, 300, 128, 3, 0], 6, 2, 96, F16, causal)


def test_empty_sequences():
    check([0, 20, 0, 0, 300, 0], [0, 20, 7, 0, 300, 0], 4, 4, 64, BF16)
    q = torch.randn(3, 2, 64, device="cuda").to(BF16)
    assert (api.attend_prompt(q, q[:0], q[:0]) == 0).all() and api.attend_prompt(q[:0], q, q).shape == (0, 2, 64)


def test_many_sequences():
    counts = [(i * 37) % 91 for i in range(200)]
    check(counts, counts, 4, 1, 64, BF16)


def test_long():
    check([5000, 77], [5000, 77], 2, 1, 128, BF16)


@pytest.mark.parametrize("size,scale", [(40.0, None), (1e-3, None), (1.0, 3.0), (1.0, 1e-10)])
def test_peaked_flat_and_scaled(size, scale):
    """Scores that grow and fall by hundreds along a row: the maximum is replaced now and then."""
    for dtype in (BF16, F16):
        check([700], [700], 2, 1, 128, dtype, size=size, scale=scale)


def test_growing_scores():
    """Keys in an order that makes every block's scores larger than the last one's, and smaller; by little and by much."""
    for step in (0.01, 0.2, 5.0):
        for sign in (1, -1):
            q = torch.zeros(256, 2, 64, dtype=BF16, device="cuda")
            q[..., 0] = 1
            k = torch.randn(1500, 1, 64, device="cuda").to(BF16)
            k[:, 0, 0] = (sign * step * torch.arange(1500, device="cuda") * 0.1).to(BF16)
            v = torch.randn(1500, 1, 64, device="cuda").to(BF16)
            out = api.attend_prompt(q, k, v, causal=True, scale=1.0, starts=ints([0, 256]), starts_k=ints([0, 1500]))
            want, far = reference(q, k, v, True, 1.0)
            assert ((out.double() - want).abs() <= far).all()


def test_one_sequence_without_starts_and_default_starts():
    q, k = torch.randn(333, 8, 128, device="cuda").to(F16), torch.randn(333, 4, 128, device="cuda").to(F16)
    out = api.attend_prompt(q, k, k)
    assert torch.equal(out, api.attend_prompt(q, k, k, ints([0, 333])))
    want, far = reference(q, k, k)
    assert ((out.double() - want).abs() <= far).all()
    # heads before tokens in memory, heads that are one and the same
    assert torch.equal(out, api.attend_prompt(q.transpose(0, 1).contiguous().transpose(0, 1), k, k))
    one = k[:, :1]
    assert torch.equal(api.attend_prompt(q, one.expand(333, 4, 128), one.expand(333, 4, 128)), api.attend_prompt(q, one.repeat(1, 4, 1), one.repeat(1, 4, 1)))


def test_nan_of_one_sequence_reaches_no_other():
    q, k, v = (torch.randn(400, h, 128, device="cuda").to(BF16) for h in (4, 2, 2))
    good = api.attend_prompt(q, k, v, ints([0, 130, 300, 400]))
    k[140], v[150], q[160] = math.nan, math.inf, math.nan
    out = api.attend_prompt(q, k, v, ints([0, 130, 300, 400]))
    assert torch.equal(out[:130], good[:130]) and torch.equal(out[300:], good[300:]) and torch.isnan(out[160:300]).all()
    assert torch.equal(out[130:140], good[130:140]) or torch.isnan(out[130:140]).any()      # the same tile: may be reached by the value


def test_starts_in_disorder_touch_nothing_else():
    q = torch.randn(50, 4, 64, device="cuda").to(BF16)
    room = torch.full((52, 4, 64), GUARD, dtype=BF16, device="cuda")
    for starts in ([0, 50, 0, 50], [50, 4, 2, 0], [-5, 3, 100, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31, 0, 1]):
        for starts_k in ([0, 50, 0, 50], [2 ** 31 - 1, -2 ** 31, 7, 2 ** 31 - 1]):
            api.attend_prompt(q, q, q, ints(starts), ints(starts_k), out=room[1:51])
    api.bs_check_status()
    assert (room[0] == GUARD).all() and (room[51] == GUARD).all()


def test_streams_and_graphs():
    """Calls on named streams, two at once, and a captured one that is replayed with other prompts and starts; the same bits every time."""
    q, k, v = (torch.randn(1000, h, 128, device="cuda").to(BF16) for h in (8, 2, 2))
    starts = ints([0, 300, 1000])
    want = api.attend_prompt(q, k, v, starts).clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [api.attend_prompt(q, k, v, starts, stream=s) for _ in range(10) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = api.attend_prompt(q, k, v, starts)
    for cut in (0, 1, 500, 999, 1000):
        starts.copy_(torch.tensor([0, cut, 1000], dtype=torch.int32))
        q.copy_(torch.randn(1000, 8, 128))
        g.replay()
        for i, j in ((0, cut), (cut, 1000)):
            ref, far = reference(q[i:j], k[i:j], v[i:j])
            assert ((out[i:j].double() - ref).abs() <= far).all()


def test_a_prompt_then_tokens_then_eviction():
    """As a program uses them: prompts attended to and stored, tokens decoded over the cache, sequences cut, decoded on."""
    import kv4_reference as ref4
    H, Hq, D, lens = 2, 8, 128, [200, 75]
    gen = torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=gen).to(BF16)  # noqa: E731
    cache, table = api.cache_kv4(20, H, D, page=32), torch.randperm(20, generator=gen).view(2, 10).int().cuda()
    q, k, v = rand(275, Hq, D).cuda(), rand(275, H, D).cuda(), rand(275, H, D).cuda()
    starts, lengths = starts_of(lens), ints(lens)
    out = api.attend_prompt(q, k, v, starts)
    for i, n in ((0, 200), (200, 75)):
        want, far = reference(q[i:i + n], k[i:i + n], v[i:i + n])
        assert ((out[i:i + n].double() - want).abs() <= far).all()
    api.append_kv4(k, v, cache, table, ints([0, 0]), starts)
    held = [[x[:200].cpu(), x[200:].cpu()] for x in (k, v)]
    weights = torch.zeros(2, H, 320, device="cuda")
    summed = [torch.zeros(H, 320, dtype=torch.float64) for _ in range(2)]
    for step in range(12):
        if step == 6:
            lengths, weights, kept = api.evict_kv4(cache, table, lengths, weights, 64, recent=16)
            assert lengths.tolist() == [64, 64]
            for b in range(2):
                at = kept[b].cpu().long()
                held = [[x.gather(0, at.T.unsqueeze(-1).expand(-1, -1, D)) if c == b else x for c, x in enumerate(part)] for part in held]
                summed[b] = torch.cat([summed[b].gather(1, at), torch.zeros(H, 256, dtype=torch.float64)], 1)
        tq, tk, tv = rand(2, Hq, D), rand(2, H, D), rand(2, H, D)
        api.append_kv4(tk.cuda(), tv.cuda(), cache, table, lengths)
        lengths = lengths + 1
        out = api.attend_kv4(tq.cuda(), cache, table, lengths, weights=weights)
        for b in range(2):
            held[0][b], held[1][b] = torch.cat([held[0][b], tk[b:b + 1]]), torch.cat([held[1][b], tv[b:b + 1]])
            want, far, got, _ = ref4.attend(tq[b:b + 1], held[0][b], held[1][b], D)
            assert ((out[b:b + 1].cpu().double() - want).abs() <= far).all()
            summed[b][:, :got.shape[1]] += got
    assert lengths.tolist() == [70, 70]
    assert torch.allclose(weights.cpu().double(), torch.stack(summed), atol=1e-4)
    api.bs_check_status()


def test_refusals():
    q, k = torch.zeros(4, 4, 64, dtype=BF16, device="cuda"), torch.zeros(4, 2, 64, dtype=BF16, device="cuda")
    s = ints([0, 4])
    for bad in (lambda: api.attend_prompt(q.float(), k.float(), k.float()), lambda: api.attend_prompt(q, k.half(), k), lambda: api.attend_prompt(q, k, k[:3]), lambda: api.attend_prompt(q[0], k, k),
                lambda: api.attend_prompt(q[:, :3], k, k), lambda: api.attend_prompt(q[..., :32], k, k), lambda: api.attend_prompt(q, k, k[:, :1]), lambda: api.attend_prompt(q, k, k, s.long()),
                lambda: api.attend_prompt(q, k, k, s, ints([0, 2, 4])), lambda: api.attend_prompt(q, k, k, ints([0])), lambda: api.attend_prompt(q, k, k, None, s), lambda: api.attend_prompt(q, k, k, s, out=q),
                lambda: api.attend_prompt(q, k, k, out=q[:3].clone()), lambda: api.attend_prompt(q.cpu(), k, k), lambda: api.attend_prompt(q, k.clone().requires_grad_(), k),
                lambda: api.attend_prompt(q, k, k, s.cpu())):
        with pytest.raises(ValueError):
            bad()
    z = torch.zeros(4 * 4 * 136 + 8, dtype=BF16, device="cuda")
    for bad in (lambda: api.attend_prompt(q, k, k, scale=0.0), lambda: api.attend_prompt(q, k, k, scale=-2.0), lambda: api.attend_prompt(q, k, k, scale=math.inf),
                lambda: api.attend_prompt(z[:2176].view(4, 4, 136), z[:2176].view(4, 4, 136), z[:2176].view(4, 4, 136)),
                lambda: api.attend_prompt(z[:4 * 129 * 4].view(4, 129, 4), z[:16].view(4, 1, 4), z[:16].view(4, 1, 4)),
                lambda: api.attend_prompt(z[1:1 + 1024].view(4, 4, 64), k, k)):
        with pytest.raises(BitserialError):
            bad()
