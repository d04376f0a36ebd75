"""Keys and values of 4 bits on the GPU where the kernels' arithmetic is at its ends, against their definitions in 64 bits."""
import math

import pytest
import torch

import kv4_reference as ref
from paper_2207_08820_b200 import api
from paper_2207_08820_b200._lib import BitserialError
from test_gpu_kv4 import BF16, F16, Filled, ints, same, starts_of, weights_of

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------------- the quantiser

def stored(x, group):
    """What the cache gives back for vectors x [n, 1, D], as keys and as values."""
    n, _, D = x.shape
    cache, table = api.cache_kv4(-(-n // 256), 1, D, page=256, group=group, dtype=x.dtype), torch.arange(-(-n // 256), dtype=torch.int32, device="cuda").unsqueeze(0)
    api.append_kv4(x.cuda(), x.cuda(), cache, table, ints([0]), ints([0, n]))
    return [y.cpu() for y in api.read_kv4(cache, table, ints([0]), ints([0, n]), total=n)]


def read(x, group):
    """As kv4_reference.read, where a difference from the offset takes more than the 53 bits of a double as well: what its rounding lost decides on which side of a
    border the quotient is."""
    v = x.double().unflatten(-1, (-1, group))
    _, step, lo = (y.unsqueeze(-1) if y.dim() < v.dim() else y for y in ref.quantise(x, group))
    d = v - lo
    back = v - d
    lost = (v - (d + back)) + (back - lo)
    c = torch.floor(d / step)
    rest = d - c * step - step / 2          # exact beside a border
    c = torch.where((rest > 0) | ((rest == 0) & ((lost > 0) | ((lost == 0) & (c % 2 == 1)))), c + 1, c).clamp(0, 15)
    return (c * step + lo).flatten(-2).float().to(x.dtype)


def test_differences_that_take_25_bits():
    """A quotient of 8.50000047 whose difference, rounded to binary32, lies on the border below it."""
    x = torch.full((1, 1, 64), 35296.0, dtype=F16)
    x[0, 0, ::32], x[0, 0, 1::32] = 2047 / 512, 62272.0
    codes, steps, _ = ref.quantise(x, 32)
    assert steps[0, 0, 0] == 4152 and codes[0, 0, 0, 2] == 9
    for back in stored(x, 32):
        assert same(back, ref.read(x, 32)) and same(back, read(x, 32))


@pytest.mark.parametrize("few", [True, False], ids=["few", "many"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_borders_beside_small_offsets(dtype, few):
    """Offsets of all magnitudes, with all ones in their mantissas, and values next to every border."""
    bits = 8 if dtype == BF16 else 11
    gen = torch.Generator().manual_seed(5)
    n = 300 if few else 40000
    span = 60000 * (0.25 + 0.75 * torch.rand(n, generator=gen).double())
    least = torch.exp2(-torch.randint(0, 24, (n,), generator=gen).double()) * span.log2().floor().exp2() * (2 - 2.0 ** (1 - torch.randint(1, bits + 1, (n,), generator=gen).double()))
    least = torch.where(least < span / 4, least, span / 4) * (torch.randint(0, 2, (n,), generator=gen) * 2 - 1)
    least, span = least.to(dtype).double(), span.to(dtype).double()
    most = torch.where(least + span < 65000, span, span / 2).to(dtype).double()
    step = ((most - least).float() / torch.full((n,), 15.0)).to(dtype).double()
    near = (torch.arange(15) + 0.5) * step.unsqueeze(1) + least.unsqueeze(1)
    low = near.to(dtype)
    ulp = torch.exp2(torch.floor(torch.log2(low.double().abs().clamp(min=1e-30)))) * torch.finfo(dtype).eps
    other = (low.double() + torch.where(near > low.double(), ulp, -ulp)).to(dtype)        # the neighbour on the far side of the border
    x = torch.cat([least.unsqueeze(1).to(dtype), most.unsqueeze(1).to(dtype), low, other], 1)
    x = torch.where((x.double() < least.unsqueeze(1)) | (x.double() > most.unsqueeze(1)), least.unsqueeze(1).to(dtype), x)
    x = torch.cat([x, x.flip(1)], 1).unsqueeze(1)
    for back in stored(x, 32):
        assert same(back, read(x, 32))



# --------------------------------------------------------------------------------------------------------------------- attention

def check(f, q, counts, scale=None, weights=False, reference=ref.attend):
    """Attention of packed queries over a filled cache against a definition."""
    w = torch.zeros(len(counts), f.H, max(f.lengths), device="cuda") if weights else None
    out = api.attend_kv4(q.cuda(), f.cache, f.table, ints(f.lengths), starts_of(counts), scale=scale, weights=w).cpu().double()
    i = 0
    for b, t in enumerate(counts):
        want, far, got, got_far = reference(q[i:i + t], f.k[b], f.v[b], f.group, scale)
        off = (out[i:i + t] - want).abs()
        assert (off <= far).all(), (b, off.max(), (off / far).max())
        if weights:
            assert ((w[b, :, :f.lengths[b]].cpu().double() - got).abs() <= got_far + 2.0 ** -23).all()
        i += t


@pytest.mark.parametrize("scale", [1e-44, 1e-38, 1e-30, 1e-20, 1e-15, 1e20, 1e31, 2e31, 1e35, 2.3e38])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_scales_near_the_ends_of_binary32(dtype, scale):
    """Queries of zeros see the mean of the values whatever the scale is, and so do all where the scale leaves nothing of the scores; one that is large picks entries."""
    f = Filled(30, [77, 300, 1], 2, 64, 16, 32, dtype)
    q = torch.zeros(30, 6, 64, dtype=dtype)
    check(f, q, [14, 15, 1], scale, weights=True)
    if scale < 1:
        q[::2] = torch.randn(15, 6, 64, generator=torch.Generator().manual_seed(1)).to(dtype)
        check(f, q, [14, 15, 1], scale, weights=True)


@pytest.mark.parametrize("power", [-110, -105, -100, -60, 60, 100, 105])
def test_scales_that_make_up_for_the_size_of_queries(power):
    """Scores of ordinary size out of products that are none."""
    f = Filled(31, [77, 300], 2, 128, 64, 64, BF16)
    q = (torch.randn(9, 6, 128, generator=torch.Generator().manual_seed(2)) * 2.0 ** power).to(BF16)
    q[3] = 0
    check(f, q, [4, 5], 2.0 ** -power / 128 ** 0.5, weights=True)


@pytest.mark.parametrize("keys,scale", [(1.0, None), (6000.0, None), (1e-4, 1e20)])
def test_keys_and_scales(keys, scale):
    f = Filled(32, [200], 1, 64, 64, 64, F16, spread=keys * 0.1)
    check(f, torch.zeros(3, 4, 64, dtype=F16), [3], scale)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("size", [1e-1, 1e-2, 1e-3, 1e-4, 1e-5, 1e-6, 5e-7])
def test_small_queries(size, dtype):
    """Queries far below one with a scale that makes up for it: no bits are lost on the way."""
    f = Filled(33, [500, 40], 2, 128, 64, 128, dtype)
    q = (torch.randn(7, 8, 128, generator=torch.Generator().manual_seed(3)) * size).to(dtype)
    q[4:] = torch.where(torch.arange(128) % 2 == 0, q[4:], q[4:] / 64)
    check(f, q, [4, 3], 1 / (size * 128 ** 0.5), weights=True)


@pytest.mark.parametrize("size,keys,scale", [(3e-6, 6000.0, 5.0), (5e-7, 6000.0, 28.0), (1e-4, 10000.0, None), (6e4, 1.0, 1e-5)])
def test_fp16_queries_and_keys_far_apart(size, keys, scale):
    f = Filled(34, [300], 1, 128, 64, 64, F16, fill=False)
    gen = torch.Generator().manual_seed(4)
    f.k[0] = (torch.rand(300, 1, 128, generator=gen) * keys).to(F16)
    api.append_kv4(f.k[0].cuda(), f.v[0].cuda(), f.cache, f.table, ints([0]), ints([0, 300]))
    q = ((torch.rand(2, 4, 128, generator=gen) * 2 - 1) * size).to(F16)
    check(f, q, [2], scale)


def attend_by_group(q, k, v, group, scale=None):
    """As kv4_reference.attend, but what the products of weights and steps lose below fp16's range counts against the largest such product of the same row and group
    of channels: half of fp16's last place, 2^-25 of it, for each entry's code up to 15."""
    out, far, got, got_far = ref.attend(q, k, v, group, scale)
    (t, Hq, D), (n, H) = q.shape, k.shape[:2]
    scale = D ** -0.5 if scale is None else scale
    vp, vs = ref.parts(v, group)        # [n, H, D], [n, H, groups]
    (kp, _), kk, vv = ref.parts(k, group), ref.values(k, group), ref.values(v, group)
    for j in range(Hq):
        h = j // (Hq // H)
        a = scale * (q[:, j].double() @ kk[:, h].T)
        seen = torch.arange(n) <= (n - t + torch.arange(t)).unsqueeze(1)
        p = torch.where(seen.any(1, keepdim=True), torch.softmax(torch.where(seen, a, -math.inf), 1), 0.0)
        size = scale * (q[:, j].double().abs() @ kp[:, h].T)
        off = size * (D / 16 + 8) * 2.0 ** -23 + 2.0 ** -34 * scale * q[:, j].double().abs().amax(1, keepdim=True) * kp[:, h].sum(1)
        # what a row does not attend to may be as far off as it is: entries count by the weights that they may have
        most = p * torch.exp(2 * off.clamp(max=50))
        mean = (most * off).sum(1, keepdim=True)
        weight = p * (2 * torch.expm1((off + mean + 6 * 2.0 ** -24 * size).clamp(max=50)) + 2.0 ** -19 + (n / 16 + 16) * 2.0 ** -24 + (2.0 ** -22 if q.dtype == F16 else 2.0 ** -11))
        largest = (p.unsqueeze(-1) * vs[:, h]).amax(1)        # [t, groups]
        lost = n * 15 * 2.0 ** -25 * 2 * largest.repeat_interleave(group, 1)
        bound = weight @ vp[:, h] + lost
        far[:, j] = bound + ref.HALF[q.dtype] * (out[:, j].abs() + bound) + torch.finfo(q.dtype).smallest_normal * torch.finfo(q.dtype).eps
    return out, far, got, got_far


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("power", [4, 10, 14, 16])
@pytest.mark.parametrize("where", ["first", "last", "among"])
def test_large_values_that_get_no_attention(where, power, dtype):
    """Entries whose values are far larger than the others', and whose scores leave them no weight: the others lose nothing by them."""
    n, D = 400, 128
    f = Filled(35, [n], 1, D, 64, 128, dtype, fill=False)
    gen = torch.Generator().manual_seed(power)
    q = torch.randn(3, 4, D, generator=gen)
    q[..., 0] = 4.0
    f.k[0][:, 0, 0] = 0
    f.v[0] = (torch.randn(n, 1, D, generator=gen) * 2.0 ** -6).to(dtype)
    at = {"first": slice(0, 3), "last": slice(n - 6, n - 3), "among": slice(5, n, 37)}[where]
    f.k[0][at, 0, 0] = -400.0
    f.v[0][at] = (torch.randn(f.v[0][at].shape, generator=gen) * 2.0 ** (power - 6)).to(dtype)
    api.append_kv4(f.k[0].cuda(), f.v[0].cuda(), f.cache, f.table, ints([0]), ints([0, n]))
    check(f, q.to(dtype), [3], reference=attend_by_group)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("D,group", [(64, 32), (96, 32), (128, 32), (128, 64)])
def test_groups_of_channels_of_other_sizes(D, group, dtype):
    """Values whose groups of channels are powers of two apart, the smallest 2^-14 of the largest."""
    f = Filled(36, [300, 33], 2, D, 16, group, dtype, fill=False)
    groups = D // group
    size = torch.exp2(torch.linspace(0, -14, groups)).repeat_interleave(group)
    f.v = [(v.float() * size).to(dtype) for v in f.v]
    api.append_kv4(torch.cat(f.k).cuda(), torch.cat(f.v).cuda(), f.cache, f.table, ints([0, 0]), starts_of([300, 33]))
    q = torch.randn(8, 6, D, generator=torch.Generator().manual_seed(9)).to(dtype)
    check(f, q, [5, 3], reference=attend_by_group)


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("step", [0.5, 3.0, 20.0, 300.0])
def test_scores_and_values_that_climb_apart(step, order):
    """Scores that grow along the sequence while the values shrink by as much or more, and the other way round."""
    n = 600
    f = Filled(37, [n], 1, 64, 32, 64, BF16, fill=False)
    gen = torch.Generator().manual_seed(6)
    q = torch.zeros(2, 3, 64)
    q[..., 0] = 1.0
    f.k[0] = torch.randn(n, 1, 64, generator=gen).to(BF16)
    f.k[0][:, 0, 0] = (order * step * torch.arange(n) / 16).to(BF16)
    for slope in (-1, 1):
        f.v[0] = (torch.randn(n, 1, 64, generator=gen) * torch.exp2(slope * 90 * (torch.arange(n) / n - 0.5)).view(-1, 1, 1)).to(BF16)
        api.append_kv4(f.k[0].cuda(), f.v[0].cuda(), f.cache, f.table, ints([0]), ints([0, n]))
        check(f, q.to(BF16), [2], 1.0, reference=attend_by_group)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("power,gap", [(4, 1), (16, 1), (20, 1), (22, 1), (24, 4), (26, 16), (28, 64)])
def test_large_scores(power, gap, order, dtype):
    """Scores of the same large part each, and whole numbers of gaps that set them apart."""
    n, D = 600, 64
    gen = torch.Generator().manual_seed(7)
    f = Filled(44, [n], 1, D, 32, 32, dtype, fill=False)
    steps = torch.arange(n) // 40 if order != "mixed" else torch.randint(0, 16, (n,), generator=gen)
    steps = 15 - steps if order == "down" else steps
    steps[:2], steps[-2:] = 0, 15 if order == "up" else 0
    f.k[0] = torch.zeros(n, 1, D, dtype=dtype)
    f.k[0][:, 0, 0], f.k[0][:, 0, 33], f.k[0][:, 0, 34] = 15 * 2.0 ** (power - power // 2 - 4), (gap * steps).to(dtype), 15 * gap         # codes are exact
    api.append_kv4(f.k[0].cuda(), f.v[0].cuda(), f.cache, f.table, ints([0]), ints([0, n]))
    q = torch.zeros(6, 3, D, dtype=dtype)
    q[..., 0], q[..., 33] = 2.0 ** (power // 2), 1.0
    q[::2, :, 0] *= -1
    k = ref.values(f.k[0], 32)[:, 0]
    assert torch.equal(k[:, 33], gap * steps.double()) and (k[:, 0] == k[0, 0]).all()
    seen = torch.arange(n) <= (n - 6 + torch.arange(6)).unsqueeze(1)
    p = torch.softmax(torch.where(seen, gap * steps.double(), -math.inf), 1)
    v, vs = ref.values(f.v[0], 32)[:, 0], ref.parts(f.v[0], 32)[1][:, 0].repeat_interleave(32, 1)
    out = api.attend_kv4(q.cuda(), f.cache, f.table, ints([n]), ints([0, 6]), scale=1.0).cpu().double()
    # distances of up to 15 gaps, of those that leave a weight: 2^-17 of it, and the exponential; a weight times a step in fp16, one or two terms; sums; the output's rounding
    part = ref.parts(f.v[0], 32)[0][:, 0]
    bound = (2.0 ** -16 + (2.0 ** -11 if dtype == BF16 else 2.0 ** -22) + (n / 16 + 16) * 2.0 ** -24) * (p @ part) + n * 15 * 2.0 ** -25 * 2 * (p.unsqueeze(-1) * vs).amax(1)
    want = (p @ v).unsqueeze(1)
    far = bound.unsqueeze(1) + ref.HALF[dtype] * (want.abs() + bound.unsqueeze(1))
    assert ((out - want).abs() <= far).all(), ((out - want).abs().max(), ((out - want).abs() / far).max())


# --------------------------------------------------------------------------------------------------------------------- eviction

def evict_around(w, n, keep, recent, there, places):
    """Where each place's entry was, of one head: what stays of the entries that are there takes the places that are."""
    entries = [i for i in range(n) if there(i)]
    stay = min(len(entries), len(places))
    if len(entries) > stay:
        new = min(recent, stay)
        old, new = entries[:len(entries) - new], entries[len(entries) - new:]
        first = torch.isnan(w[old])
        order = sorted(range(len(old)), key=lambda j: (not bool(first[j]), -float(torch.nan_to_num(w[old[j]], nan=0.0, posinf=math.inf, neginf=-math.inf)), j))
        entries = sorted(old[j] for j in order[:stay - len(new)]) + new
    return dict(zip(places, entries))


HOLES = {"front": lambda p, n: p < 2, "middle": lambda p, n: p in (1, 3, 4), "end": lambda p, n: p >= n - 1, "all": lambda p, n: True, "every other": lambda p, n: p % 2 == 0}


@pytest.mark.parametrize("inside", [True, False], ids=["inside", "into"])
@pytest.mark.parametrize("keep,recent", [(1, 0), (40, 0), (40, 40), (100, 33), (1000, 5)])
@pytest.mark.parametrize("where", HOLES)
@pytest.mark.parametrize("kind", ["spread", "ties", "any"])
def test_evict_entries_that_are_not_there(kind, where, keep, recent, inside):
    """Sequences with pages that the cache does not have, and places on such pages: what is not there does not stay, and what stays is there afterwards."""
    lengths, H, D, page = [0, 10, 40, 100, 333], 2, 64, 16
    f = Filled(40, lengths, H, D, page, 32, F16)
    B, N = len(lengths), 333
    w = weights_of(keep + recent, B, H, N, kind)
    table = f.table_cpu.clone()
    for b, n in enumerate(lengths):
        for p in range(-(-n // page)):
            if HOLES[where](p, -(-n // page)):
                table[b, p] = -1 if b % 2 else 10 ** 9
    cache, into = f.cache, None
    if not inside:
        wide = -(-min(keep, N) // page)
        cache = api.cache_kv4(f.cache.data.shape[0] + B * wide, H, D, page=page, group=32, dtype=F16)
        cache.data.fill_(255)
        cache.data[:f.cache.data.shape[0]] = f.cache.data
        into = (f.cache.data.shape[0] + torch.randperm(B * wide, generator=torch.Generator().manual_seed(1))).view(B, wide).int()
        if wide > 2:
            into[3, 1], into[4, 0] = -5, cache.data.shape[0]
    n_out, w_out, kept = api.evict_kv4(cache, table.cuda(), ints(lengths), w.cuda(), keep, recent=recent, into=None if inside else into.cuda())
    target = table if inside else into
    q = torch.randn(B, 2 * H, D, generator=torch.Generator().manual_seed(2)).to(F16)
    seen = api.attend_kv4(q.cuda(), cache, target.cuda(), n_out).cpu().double()
    pages = cache.data.shape[0]
    for b, n in enumerate(lengths):
        there = lambda i: 0 <= int(table[b, i // page]) < pages  # noqa: E731
        places = [r for r in range(min(keep, N, target.shape[1] * page)) if 0 <= int(target[b, r // page]) < pages]
        for h in range(H):
            if inside and n <= keep:        # as they are
                want = {r: r for r in range(n)}
            else:
                want = evict_around(w[b, h], n, keep, recent, there, places)
            assert int(n_out[b]) == (max(want) + 1 if want else 0), (b, h)
            assert kept[b, h].tolist() == [want.get(r, -1) for r in range(keep)], (b, h)
            assert same(w_out[b, h].cpu(), torch.tensor([float(w[b, h, want[r]]) if r in want else 0.0 for r in range(N)]))
            at = [i for r, i in sorted(want.items()) if there(i)]
            out, far, _, _ = ref.attend(q[b:b + 1, 2 * h:2 * h + 2], f.k[b][at, h:h + 1], f.v[b][at, h:h + 1], 32)
            assert ((seen[b:b + 1, 2 * h:2 * h + 2] - out).abs() <= far).all(), (b, h)


def test_evict_long_sequences_that_are_not_all_there():
    """By clusters of CTAs, one of which does the work."""
    n, keep, recent, page = 70000, 30000, 1000, 64
    f = Filled(41, [n], 2, 64, page, 64, F16)
    table = f.table_cpu.clone()
    gone = torch.rand(table.shape[1], generator=torch.Generator().manual_seed(3)) < 0.3
    table[0, gone] = -1
    w = weights_of(5, 1, 2, n, "ties")
    into = torch.arange(f.cache.data.shape[0], f.cache.data.shape[0] + -(-keep // page), dtype=torch.int32).unsqueeze(0)
    cache = api.cache_kv4(f.cache.data.shape[0] + into.shape[1], 2, 64, page=page, dtype=F16)
    cache.data[:f.cache.data.shape[0]] = f.cache.data
    n_out, w_out, kept = api.evict_kv4(cache, table.cuda(), ints([n]), w.cuda(), keep, recent=recent, into=into.cuda())
    entries = torch.arange(n)[~gone.repeat_interleave(page)[:n]]
    k, _ = api.read_kv4(cache, into.cuda(), ints([0]), ints([0, keep]), total=keep)
    assert n_out.tolist() == [keep]
    for h in range(2):
        old = entries[:-recent]
        best = old[torch.sort(w[0, h, old], descending=True, stable=True).indices[:keep - recent]].sort().values
        want = torch.cat([best, entries[-recent:]])
        assert torch.equal(kept[0, h].cpu().long(), want) and same(w_out[0, h, :keep].cpu(), w[0, h, want])
        assert same(k[:, h].cpu(), ref.read(f.k[0][want, h], 64))


def test_weights_in_any_order():
    """Weights [heads, sequences, entries] as well as [sequences, heads, entries], added to and read; rows that lie over one another are refused."""
    f = Filled(42, [70, 200, 33], 2, 64, 16, 64, BF16)
    q, lengths = torch.randn(3, 6, 64, device="cuda").to(BF16), ints(f.lengths)
    plain, room = torch.zeros(3, 2, 200, device="cuda"), torch.zeros(2, 3, 210, device="cuda")
    turned = room.transpose(0, 1)[..., 5:205]
    out = api.attend_kv4(q, f.cache, f.table, lengths, weights=plain)
    assert torch.equal(out, api.attend_kv4(q, f.cache, f.table, lengths, weights=turned)) and torch.equal(plain, turned)
    assert (room[..., :5] == 0).all() and (room[..., 205:] == 0).all()
    data = f.cache.data.clone()
    first = api.evict_kv4(f.cache, f.table, lengths, turned, 20, recent=3)
    f.cache.data.copy_(data)
    assert all(same(a, b) for a, b in zip(first, api.evict_kv4(f.cache, f.table, lengths, plain, 20, recent=3)))
    for strides in ((100, 200, 1), (200, 100, 1), (0, 200, 1), (399, 200, 1)):
        with pytest.raises(ValueError):
            api.attend_kv4(q, f.cache, f.table, lengths, weights=torch.zeros(2000, device="cuda").as_strided((3, 2, 200), strides))


def test_one_row_of_pages_for_all_sequences():
    """A prefix that several sequences share, by a row of the table that is expanded and not copied: read, attended to and cut into pages of their own."""
    n, B = 100, 3
    f = Filled(43, [n], 2, 64, 16, 64, BF16)
    one, many = f.table.expand(B, -1), f.table.repeat(B, 1)
    q, lengths = torch.randn(B, 4, 64, device="cuda").to(BF16), ints([n, 40, 0])
    assert torch.equal(api.attend_kv4(q, f.cache, one, lengths), api.attend_kv4(q, f.cache, many, lengths))
    for a, b in zip(api.read_kv4(f.cache, one, ints([0, 7, 20]), ints([0, 50, 60, 80]), total=80), api.read_kv4(f.cache, many, ints([0, 7, 20]), ints([0, 50, 60, 80]), total=80)):
        assert same(a, b)
    cache = api.cache_kv4(f.cache.data.shape[0] + 6, 2, 64, page=16)
    cache.data[:f.cache.data.shape[0]] = f.cache.data
    into = torch.arange(f.cache.data.shape[0], f.cache.data.shape[0] + 6, dtype=torch.int32, device="cuda").view(3, 2)
    w = weights_of(7, B, 2, n, "ties").cuda()
    first = api.evict_kv4(cache, one, lengths, w, 20, recent=3, into=into)
    held = api.read_kv4(cache, into, ints([0, 0, 0]), ints([0, 20, 40, 40]), total=40)
    cache.data[f.cache.data.shape[0]:] = 255
    assert all(same(a, b) for a, b in zip(first, api.evict_kv4(cache, many, lengths, w, 20, recent=3, into=into)))
    assert all(same(a, b) for a, b in zip(held, api.read_kv4(cache, into, ints([0, 0, 0]), ints([0, 20, 40, 40]), total=40)))
    k, v = torch.randn(B, 2, 64, device="cuda").to(BF16), torch.randn(B, 2, 64, device="cuda").to(BF16)
    api.append_kv4(k, v, f.cache, one, ints([3, 50, 99]))
    back = api.read_kv4(f.cache, many, ints([3, 50, 99]))
    assert same(back[0].cpu(), ref.read(k.cpu(), 64)) and same(back[1].cpu(), ref.read(v.cpu(), 64))
    with pytest.raises(BitserialError):
        api.evict_kv4(f.cache, one, lengths, w, 20)
