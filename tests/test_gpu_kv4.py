"""Keys and values of 4 bits on the GPU: stored, read back, attended to and evicted, against their definitions in 64 bits (kv4_reference.py)."""
import math
import re

import pytest
import torch

import kv4_reference as ref
from graph_launches import launches
from paper_2207_08820_b200 import api
from paper_2207_08820_b200._lib import BitserialError

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
GUARD = 77.0


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def starts_of(counts):
    return ints([0] + torch.tensor(counts, dtype=torch.long).cumsum(0).tolist())


class Filled:
    """A cache with sequences of given lengths, whatever else it holds being NaN, their pages in random order between pages that nobody has."""

    def __init__(self, seed, lengths, H, D, page, group, dtype, room=0, spread=1.0, fill=True):
        gen = torch.Generator().manual_seed(seed)
        self.lengths, self.H, self.D, self.page, self.group, self.dtype = lengths, H, D, page, group, dtype
        wide = max(1, max(-(-n // page) for n in lengths)) + room
        pages = len(lengths) * wide + 3
        self.cache = api.cache_kv4(pages, H, D, page=page, group=group, dtype=dtype)
        self.cache.data.fill_(255)
        self.table_cpu = torch.randperm(pages, generator=gen)[:len(lengths) * wide].view(len(lengths), wide).int()
        self.table = self.table_cpu.cuda()
        rand = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        self.k = [((rand(n, H, D) * torch.exp(0.5 * rand(H, D)) + rand(H, D)) * spread).to(dtype) for n in lengths]
        self.v = [(rand(n, H, D) * torch.exp(0.5 * rand(n, 1, 1))).to(dtype) for n in lengths]
        if fill and sum(lengths):
            api.append_kv4(torch.cat(self.k).cuda(), torch.cat(self.v).cuda(), self.cache, self.table, ints([0] * len(lengths)), starts_of(lengths))


def same(a, b):
    """Equal bit for bit, NaN counting as one value."""
    return torch.equal(torch.where(torch.isnan(a), 3e4, a.float()), torch.where(torch.isnan(b), 3e4, b.float()))


LAYOUTS = [(128, 64, 128), (128, 16, 32), (128, 1024, 64), (96, 32, 96), (96, 16, 32), (64, 128, 64), (64, 16, 32)]


# ------------------------------------------------------------------------------------------------------------------- the cache

@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("D,page,group", LAYOUTS)
def test_store_and_read(D, page, group, dtype):
    f = Filled(1, [0, 1, 15, 16, 17, 100, 259], 3, D, page, group, dtype)
    k, v = api.read_kv4(f.cache, f.table, ints([0] * 7), starts_of(f.lengths), total=sum(f.lengths))
    assert same(k.cpu(), ref.read(torch.cat(f.k), group)) and same(v.cpu(), ref.read(torch.cat(f.v), group))
    # single entries, and stretches from anywhere
    k, v = api.read_kv4(f.cache, f.table[3:], ints([15, 3, 99, 130]))
    for i, (b, e) in enumerate([(3, 15), (4, 3), (5, 99), (6, 130)]):
        assert same(k[i].cpu(), ref.read(f.k[b][e], group)) and same(v[i].cpu(), ref.read(f.v[b][e], group))
    k, _ = api.read_kv4(f.cache, f.table[6:], ints([101]), ints([0, 40]), total=40)
    assert same(k.cpu(), ref.read(f.k[6][101:141], group))


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_append_writes_its_entries_alone(dtype):
    """Token by token beside neighbours in the same tiles, out of the views of a fused projection; nothing else of the cache changes."""
    H, D, group = 2, 96, 32
    f = Filled(2, [30, 5, 47], H, D, 16, group, dtype, room=1)
    before = f.cache.data.clone()
    fused = torch.randn(3, 7, 3 * H, D, device="cuda").to(dtype)
    k, v = fused[:, 4, H:2 * H], fused[:, 4, 2 * H:]
    assert not k.is_contiguous()
    api.append_kv4(k, v, f.cache, f.table, ints([30, 5, 47]))
    for b, n in enumerate((30, 5, 47)):
        gk, gv = api.read_kv4(f.cache, f.table[b:b + 1], ints([0]), ints([0, n + 1]), total=n + 1)
        assert same(gk.cpu(), ref.read(torch.cat([f.k[b], k[b:b + 1].cpu()]), group)) and same(gv.cpu(), ref.read(torch.cat([f.v[b], v[b:b + 1].cpu()]), group))
    # an entry is H * (D + 8 * groups) bytes
    assert (f.cache.data != before).sum() <= 3 * H * (D + 8 * (D // group))


def test_quantiser_ties_and_extremes():
    """Quotients on ties and beside them by less than a float tells apart, groups of one value, spans near the ends of the type, infinities and NaN."""
    rows = []
    for dtype, s in ((BF16, 0.75), (BF16, 2.0 ** -100), (BF16, 1.5 * 2.0 ** 90), (F16, 0.75), (F16, 2.0 ** -20)):
        row = torch.zeros(32, dtype=torch.float64)
        row[1] = 15 * s
        for i in range(15):
            row[2 + i] = (i + 0.5) * s
            row[17 + i] = ((i + 0.5) * s) * (1 + (2 * (i % 2) - 1) * torch.finfo(dtype).eps)
        rows += [(dtype, row), (dtype, -row)]
    # the offset is far from the other values: x - m is rounded in binary32, and lies on a border afterwards
    row = torch.zeros(32, dtype=torch.float64)
    row[0], row[1] = -0.25, 7.25
    row[2], row[3] = 2.0 ** -40, -2.0 ** -40
    rows.append((BF16, row))
    for values in ([0.0], [1.0], [-3.0], [65504.0, -65504.0], [6e-8, 0.0], [1.0, math.inf], [math.nan, 2.0], [-math.inf, 0.0]):
        rows.append((F16, torch.tensor(values, dtype=torch.float64).repeat(32)[:32]))
    for values in ([3e38, -3e38], [1e-40, 0.0], [3e38, 1e38], [1e-38, -1e-38]):
        rows.append((BF16, torch.tensor(values, dtype=torch.float64).repeat(32)[:32]))
    for dtype in (BF16, F16):
        x = torch.stack([r for t, r in rows if t == dtype]).to(dtype)
        x = torch.cat([x, x.flip(1)], 1).unsqueeze(1)          # 64 channels, two groups
        n = x.shape[0]
        cache = api.cache_kv4(2, 1, 64, page=32, group=32, dtype=dtype)
        api.append_kv4(x.cuda(), x.flip(0).cuda(), cache, ints([[1, 0]]), ints([0]), ints([0, n]))
        k, v = api.read_kv4(cache, ints([[1, 0]]), ints([0]), ints([0, n]), total=n)
        assert same(k.cpu(), ref.read(x, 32)) and same(v.cpu(), ref.read(x.flip(0), 32))


def test_entries_that_are_nowhere():
    """Behind the table, before it, on pages that the cache does not have, and tokens that no sequence holds: not stored, read as zeros."""
    f = Filled(3, [20, 20], 1, 64, 16, 64, BF16)
    before = f.cache.data.clone()
    x = torch.ones(6, 1, 64, dtype=BF16, device="cuda")
    api.append_kv4(x[:2], x[:2], f.cache, f.table, ints([32, -1]))
    api.append_kv4(x[:2], x[:2], f.cache, f.table, ints([2 ** 31 - 1, -2 ** 31]))
    api.append_kv4(x[:2], x[:2], f.cache, ints([[-1, -1], [f.cache.data.shape[0], 2 ** 31 - 1]]), ints([3, 20]))
    api.append_kv4(x, x, f.cache, f.table, ints([32, 40]), ints([2, 4, 5]))
    api.append_kv4(x, x, f.cache, f.table, ints([0, 0]), ints([6, 3, 0]))
    assert torch.equal(f.cache.data, before)
    k, v = api.read_kv4(f.cache, ints([[-1, int(f.table_cpu[0, 1])]]), ints([14]), ints([0, 4]), total=5)
    assert (k[:2] == 0).all() and same(k[2:4].cpu(), ref.read(f.k[0][16:18], 64)) and (k[4] == 0).all() and (v[4] == 0).all()
    assert api.read_kv4(f.cache, f.table, ints([0, 0]), ints([0, 0, 0]), total=0)[0].shape == (0, 1, 64)


def test_offsets_beyond_32_bits():
    """A cache of more than 4 GB: the last pages are stored, read, attended to and moved."""
    H, D = 8, 128
    pages = (1 << 32) // (64 * H * (D + 8)) + 40
    cache = api.cache_kv4(pages, H, D)
    table = torch.arange(pages - 1, pages - 5, -1, dtype=torch.int32, device="cuda").unsqueeze(0)
    gen = torch.Generator().manual_seed(4)
    k, v, q = (torch.randn(n, h, D, generator=gen).to(BF16) for n, h in ((200, H), (200, H), (1, 2 * H)))
    api.append_kv4(k.cuda(), v.cuda(), cache, table, ints([0]), ints([0, 200]))
    back = api.read_kv4(cache, table, ints([0]), ints([0, 200]), total=200)
    assert same(back[0].cpu(), ref.read(k, D)) and same(back[1].cpu(), ref.read(v, D))
    out, far, _, _ = ref.attend(q, k, v, D)
    assert ((api.attend_kv4(q.cuda(), cache, table, ints([200])).cpu().double() - out).abs() <= far).all()
    w = torch.rand(1, H, 200, device="cuda")
    _, _, kept = api.evict_kv4(cache, table, ints([200]), w, 70, into=ints([[pages - 9, 0]]))
    moved = api.read_kv4(cache, ints([[pages - 9, 0]]), ints([0]), ints([0, 70]), total=70)
    for h in range(H):
        assert same(moved[0][:, h].cpu(), ref.read(k[kept[0, h].cpu().long(), h], D))


# --------------------------------------------------------------------------------------------------------------------- attention

def check_attend(f, counts, per, seed=5, starts=True, weights=False, scale=None, scale_q=1.0):
    gen = torch.Generator().manual_seed(seed)
    T, Hq, D, B = sum(counts), per * f.H, f.D, len(counts)
    q = (torch.randn(T, Hq, D, generator=gen) * scale_q).to(f.dtype)
    fused = torch.full((T, Hq + 3, D), math.nan, dtype=f.dtype, device="cuda")
    fused[:, 1:Hq + 1] = q.cuda()
    room = torch.full((T + 2, Hq, D), GUARD, dtype=f.dtype, device="cuda")
    most = max(1, max(f.lengths))
    w_room = torch.full((B, f.H + 1, most + 5), 0.25, device="cuda")
    w = w_room[:, :f.H, :most] if weights else None
    out = api.attend_kv4(fused[:, 1:Hq + 1], f.cache, f.table, ints(f.lengths), starts_of(counts) if starts else None, weights=w, scale=scale, out=room[1:T + 1])
    api.bs_check_status()
    assert (room[0] == GUARD).all() and (room[-1] == GUARD).all()
    i = 0
    for b, t in enumerate(counts):
        want, far, got, got_far = ref.attend(q[i:i + t], f.k[b], f.v[b], f.group, scale)
        off = (out[i:i + t].cpu().double() - want).abs()
        assert (off <= far).all(), (b, (off / far).max())
        if weights:
            n = f.lengths[b]
            off = (w_room[b, :f.H, :n].cpu().double() - 0.25 - got).abs()
            assert (off <= got_far + 2.0 ** -23).all(), (b, (off / (got_far + 2.0 ** -23)).max())
            assert (w_room[b, :f.H, n:] == 0.25).all()
        i += t
    assert (w_room[:, f.H] == 0.25).all()
    return out


# Tables that end with the longest sequence, and ones that could hold many times as much: short and long ones are cut and joined in different ways.
ROOM = pytest.mark.parametrize("room", [0, 20000], ids=["narrow", "wide"])


@ROOM
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("D,page,group", LAYOUTS)
def test_attend_single_tokens(D, page, group, dtype, room):
    """Lengths around tiles, units and runs; a group of heads that fills half a fragment."""
    f = Filled(6, [1, 2, 15, 16, 17, 63, 64, 65, 128, 129, 300, 1111], 2, D, page, group, dtype, room=room // page)
    check_attend(f, [1] * 12, 4, starts=False)


@ROOM
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("per", [1, 7, 8, 9, 16, 40])
def test_attend_grouped_heads(per, dtype, room):
    f = Filled(7, [77, 1, 530], 2, 64 if per == 40 else 128, 16, 32, dtype, room=room // 16)
    check_attend(f, [1, 1, 1], per, starts=False, weights=True)


@ROOM
@pytest.mark.parametrize("D,page,group", LAYOUTS)
def test_attend_several_tokens(D, page, group, room):
    """As many tokens as entries, more than rows of a tile, none, and one; attention of the entries."""
    f = Filled(8, [5, 70, 33, 260, 700], 2, D, page, group, BF16, room=room // page)
    check_attend(f, [5, 3, 0, 20, 1], 3, weights=True)


def test_attend_many_tokens():
    f = Filled(9, [300, 500], 1, 64, 32, 64, F16)
    check_attend(f, [300, 99], 2, weights=True)


def test_attend_long():
    f = Filled(10, [40000, 3], 1, 128, 256, 128, BF16)
    check_attend(f, [1, 1], 8, starts=False, weights=True)


@pytest.mark.parametrize("spread,scale_q,scale", [(1, 30, None), (100, 1, None), (1e-3, 1e-3, None), (1, 1, 1e-20), (1, 1, 2.0)])
def test_attend_peaked_flat_and_scaled(spread, scale_q, scale):
    f = Filled(11, [200, 900], 1, 128, 64, 64, BF16, spread=spread)
    check_attend(f, [1, 2], 5, scale_q=scale_q, scale=scale)


def test_attend_values_of_any_size():
    """Steps of the values that grow by many powers of two along the sequence, and fall, and are zero."""
    f = Filled(12, [700], 1, 128, 64, 32, BF16, fill=False)
    size = torch.exp2(torch.linspace(-100, 100, 700)).view(-1, 1, 1)
    for order in (slice(None), torch.arange(699, -1, -1)):
        f.v[0] = (torch.randn(700, 1, 128, generator=torch.Generator().manual_seed(1)) * size[order]).to(BF16)
        api.append_kv4(f.k[0].cuda(), f.v[0].cuda(), f.cache, f.table, ints([0]), ints([0, 700]))
        check_attend(f, [1], 4, starts=False)
    f.v[0] = torch.full((700, 1, 128), 2.5, dtype=BF16)
    api.append_kv4(f.k[0].cuda(), f.v[0].cuda(), f.cache, f.table, ints([0]), ints([0, 700]))
    assert (check_attend(f, [1], 4, starts=False) == 2.5).all()


@ROOM
def test_attend_nothing(room):
    """Sequences of no entries, rows that see none, tokens of no sequence."""
    f = Filled(13, [0, 2, 40], 2, 64, 16, 64, BF16, room=room // 16)
    q = torch.randn(9, 4, 64, device="cuda").to(BF16)
    out = torch.full_like(q, GUARD)
    w = torch.zeros(3, 2, 40, device="cuda")
    api.attend_kv4(q, f.cache, f.table, ints([0, 2, 40]), ints([1, 3, 7, 8]), out=out, weights=w)
    assert (out[0] == GUARD).all() and (out[8] == GUARD).all()
    assert (out[1:5] == 0).all()                    # no entries; two entries for four rows: the first two see none
    want, far, _, _ = ref.attend(q[5:7].cpu(), f.k[1], f.v[1], 64)
    assert ((out[5:7].cpu().double() - want).abs() <= far).all()
    assert torch.allclose(w.sum(-1), torch.tensor([[0.0], [2 * 2], [2]], device="cuda").expand(3, 2), atol=1e-5)
    assert (api.attend_kv4(q[:3], f.cache, f.table, ints([-5, 0, -2 ** 31])) == 0).all()
    assert api.attend_kv4(q[:0], f.cache, f.table, ints([0, 2, 40]), ints([0, 0, 0, 0])).shape == (0, 4, 64)


def test_attend_missing_pages_and_lengths_beyond_the_table():
    """What is not there does not count; nothing outside the table is taken for a page."""
    f = Filled(14, [100], 1, 128, 16, 128, BF16)
    table = f.table_cpu.clone()
    table[0, 2], table[0, 5] = -7, 10 ** 9
    q = torch.randn(1, 4, 128).to(BF16)
    stay = [i for i in range(100) if i // 16 not in (2, 5)]
    want, far, got, got_far = ref.attend(q, f.k[0][stay], f.v[0][stay], 128)
    w = torch.zeros(1, 1, 100, device="cuda")
    out = api.attend_kv4(q.cuda(), f.cache, table.cuda(), ints([100]), weights=w)
    assert ((out.cpu().double() - want).abs() <= far).all()
    assert ((w[0, 0, stay].cpu().double() - got[0]).abs() <= got_far[0] + 1e-7).all() and (w[0, 0, 32:48] == 0).all()
    # the table has 112 entries: a length beyond it is cut there
    cache = f.cache._replace(data=f.cache.data.clone())
    x = torch.randn(112, 1, 128).to(BF16)
    api.append_kv4(x.cuda(), x.cuda(), cache, f.table, ints([0]), ints([0, 112]))
    want, far, _, _ = ref.attend(q, x, x, 128)
    for n in (113, 10 ** 6, 2 ** 31 - 1):
        assert ((api.attend_kv4(q.cuda(), cache, f.table, ints([n])).cpu().double() - want).abs() <= far).all()


@ROOM
def test_starts_in_disorder_touch_nothing_else(room):
    f = Filled(15, [300, 40, 700], 2, 64, 16, 64, BF16, room=room // 16)
    q = torch.randn(8, 4, 64, device="cuda").to(BF16)
    room = torch.full((10, 4, 64), GUARD, dtype=BF16, device="cuda")
    before = f.cache.data.clone()
    for starts in ([0, 8, 0, 8], [8, 4, 2, 0], [-5, 3, 100, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31, 0, 1]):
        api.attend_kv4(q, f.cache, f.table, ints(f.lengths), ints(starts), out=room[1:9], weights=torch.zeros(3, 2, 700, device="cuda"))
    torch.cuda.synchronize()
    assert (room[0] == GUARD).all() and (room[9] == GUARD).all() and torch.equal(f.cache.data, before)


@ROOM
def test_nan_stays_where_it_belongs(room):
    """A stored NaN reaches the rows that see its entry, the values' only in its group; queries' only their own row."""
    f = Filled(16, [90, 90], 2, 128, 16, 32, F16, fill=False, room=room // 16)
    f.v[0][80, 0, 40] = math.inf
    f.k[1][3, 1, 7] = math.nan
    api.append_kv4(torch.cat(f.k).cuda(), torch.cat(f.v).cuda(), f.cache, f.table, ints([0, 0]), ints([0, 90, 180]))
    q = torch.randn(30, 4, 128).to(F16)
    q[25, 0, 0] = math.nan
    out = api.attend_kv4(q.cuda(), f.cache, f.table, ints([90, 90]), ints([0, 15, 30])).cpu()
    bad = torch.isnan(out)
    want = torch.zeros_like(bad)
    want[5:15, :2, 32:64] = True        # rows 75 + i of the first sequence that see entry 80
    want[15:, 2:] = True                # every row of the second one sees entry 3
    want[25, 0] = True
    assert torch.equal(bad, want)
    good, far, _, _ = ref.attend(q[:15], torch.nan_to_num(f.k[0]), torch.nan_to_num(f.v[0], posinf=0.0), 32)
    assert ((out[:5].double() - good[:5]).abs() <= far[:5]).all()


def test_shared_pages_strided_tables_and_repeated_calls():
    """Two sequences that begin on the same pages, a table that is a slice of a wider one; the same bits every time."""
    f = Filled(17, [256, 256], 2, 128, 64, 128, BF16, room=2)
    wide = torch.full((2, 11), -1, dtype=torch.int32, device="cuda")
    wide[:, 3:9] = f.table
    wide[1, 3:5] = wide[0, 3:5]
    f.k[1] = torch.cat([f.k[0][:128], f.k[1][128:]])
    f.v[1] = torch.cat([f.v[0][:128], f.v[1][128:]])
    f.table = wide[:, 3:9]
    first = check_attend(f, [1, 1], 4, starts=False, weights=True).clone()
    for _ in range(3):
        assert torch.equal(first, check_attend(f, [1, 1], 4, starts=False, weights=True))


@ROOM
def test_streams_and_graphs(room):
    """Calls on a named stream, two at once, and a captured step that is replayed with other lengths, queries and tables."""
    f = Filled(18, [2000, 40, 700], 2, 128, 64, 128, BF16, room=room // 64)
    lengths, q = ints(f.lengths), torch.randn(3, 8, 128, device="cuda").to(BF16)
    want = api.attend_kv4(q, f.cache, f.table, lengths).clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[api.attend_kv4(q, f.cache, f.table, lengths, stream=s) for _ in range(20)] for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for group in outs for o in group)
    graphs, held = [], []
    k, v = torch.randn(3, 2, 128, device="cuda").to(BF16), torch.randn(3, 2, 128, device="cuda").to(BF16)
    at, weights = lengths - 1, torch.zeros(3, 2, 2000, device="cuda")
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            api.append_kv4(k, v, f.cache, f.table, at)
            held.append(api.attend_kv4(q, f.cache, f.table, lengths, weights=weights))
        graphs.append(g)
    q.copy_(torch.randn(3, 8, 128).to(BF16))
    for step in ([2000, 40, 700], [1, 0, 65], [1999, 17, 3]):
        lengths.copy_(torch.tensor(step, dtype=torch.int32))
        at.copy_(lengths - 1)
        weights.zero_()
        for g in graphs:
            g.replay()
        for b, n in enumerate(step):
            if n:
                f.k[b][n - 1], f.v[b][n - 1] = k[b].cpu(), v[b].cpu()
            out, far, got, got_far = ref.attend(q[b:b + 1].cpu(), f.k[b][:n], f.v[b][:n], 128)
            for o in held:
                assert ((o[b:b + 1].cpu().double() - out).abs() <= far).all()
            assert ((weights[b, :, :n].cpu().double() - 2 * got).abs() <= 2 * got_far + 1e-6).all()


def test_which_kernels_run():
    """Short sequences in one launch of clusters, long ones and many with a second launch, attention of the entries in one more; the count of launches follows."""
    for lengths, room, names in (([500], 0, ["attend"]), ([500], 1000, ["attend", "join"]), ([500] * 40, 0, ["attend", "join"]), ([60] * 200, 0, ["attend"])):
        f = Filled(23, lengths, 4, 64, 64, 64, BF16, room=room)
        q, n = torch.randn(len(lengths), 4, 64, device="cuda").to(BF16), ints(lengths)
        for weights, more in ((None, []), (torch.zeros(len(lengths), 4, 500, device="cuda"), ["weights"])):
            got = launches(lambda: api.attend_kv4(q, f.cache, f.table, n, weights=weights))
            assert sorted(re.search(r"kv4_(attend|join|weights)_kernel", name)[1] for name, _ in got) == sorted(names + more), (len(lengths), room)
            before = api.launch_count
            api.attend_kv4(q, f.cache, f.table, n, weights=weights)
            assert api.launch_count - before == len(names + more)


# --------------------------------------------------------------------------------------------------------------------- eviction

def weights_of(seed, B, H, N, kind):
    gen = torch.Generator().manual_seed(seed)
    w = torch.exp(2 * torch.randn(B, H, N, generator=gen))
    if kind == "ties":
        w = (w * 4).round() / 4
    elif kind == "same":
        w = torch.full_like(w, 0.125)
    elif kind == "any":
        w = torch.randn(B, H, N, generator=gen)
        w[torch.rand(w.shape, generator=gen) < 0.1] = math.inf
        w[torch.rand(w.shape, generator=gen) < 0.1] = -math.inf
        w[torch.rand(w.shape, generator=gen) < 0.1] = math.nan
        w[torch.rand(w.shape, generator=gen) < 0.1] = 0.0
        w[torch.rand(w.shape, generator=gen) < 0.1] = -0.0
    return w


@pytest.mark.parametrize("kind", ["spread", "ties", "same", "any"])
@pytest.mark.parametrize("keep,recent", [(1, 0), (1, 1), (50, 0), (50, 50), (100, 31), (1000, 17)])
@pytest.mark.parametrize("inside", [False, True])
def test_evict(keep, recent, kind, inside):
    lengths = [0, 1, 50, 51, 99, 130, 1003]
    f = Filled(19, lengths, 3, 96, 16, 32, BF16)
    B, H, N = len(lengths), 3, 1010
    w = weights_of(keep + recent, B, H, N, kind)
    room = torch.full((B, H + 2, N + 3), GUARD, device="cuda")
    room[:, 1:H + 1, 2:N + 2] = w.cuda()
    if inside:
        into, cache = None, f.cache
    else:        # pages behind the others, of a cache that has room for them
        wide = -(-keep // 16)
        cache = api.cache_kv4(f.cache.data.shape[0] + B * wide, H, 96, page=16, group=32)
        cache.data.fill_(255)
        cache.data[:f.cache.data.shape[0]] = f.cache.data
        into = ints((f.cache.data.shape[0] + torch.randperm(B * wide, generator=torch.Generator().manual_seed(1))).view(B, wide).tolist())
    n_out, w_out, kept = api.evict_kv4(cache, f.table, ints(lengths), room[:, 1:H + 1, 2:N + 2], keep, recent=recent, into=into)
    where = f.table if inside else into
    for b, n in enumerate(lengths):
        stay = min(n, keep)
        assert int(n_out[b]) == stay
        k, v = api.read_kv4(cache, where[b:b + 1], ints([0]), ints([0, stay]), total=stay)
        for h in range(H):
            want = ref.evict(w[b, h], n, keep, recent)
            assert torch.equal(kept[b, h, :stay].cpu().long(), want) and (kept[b, h, stay:] == -1).all()
            assert same(w_out[b, h, :stay].cpu(), w[b, h, want]) and (w_out[b, h, stay:] == 0).all()
            assert same(k[:, h].cpu(), ref.read(f.k[b][want, h], 32)) and same(v[:, h].cpu(), ref.read(f.v[b][want, h], 32))
    if not inside:
        assert torch.equal(cache.data[:f.cache.data.shape[0]], f.cache.data)


@pytest.mark.parametrize("D,page,group", LAYOUTS)
def test_evict_layouts(D, page, group):
    f = Filled(20, [3000, 700], 2, D, page, group, F16)
    w = weights_of(3, 2, 2, 3000, "ties")
    n_out, _, kept = api.evict_kv4(f.cache, f.table, ints([3000, 700]), w.cuda(), 700, recent=99)
    assert n_out.tolist() == [700, 700]
    k, v = api.read_kv4(f.cache, f.table[:1], ints([0]), ints([0, 700]), total=700)
    for h in range(2):
        want = ref.evict(w[0, h], 3000, 700, 99)
        assert torch.equal(kept[0, h].cpu().long(), want)
        assert same(k[:, h].cpu(), ref.read(f.k[0][want, h], group)) and same(v[:, h].cpu(), ref.read(f.v[0][want, h], group))


def test_evict_long():
    w = weights_of(4, 1, 2, 150000, "ties")
    f = Filled(21, [150000], 2, 64, 256, 64, F16)
    n_out, w_out, kept = api.evict_kv4(f.cache, f.table, ints([150000]), w.cuda(), 60001, recent=1000)
    for h in range(2):
        old = w[0, h, :149000]
        best = torch.sort(old, descending=True, stable=True).indices[:59001].sort().values
        want = torch.cat([best, torch.arange(149000, 150000)])
        assert torch.equal(kept[0, h].cpu().long(), want) and torch.equal(w_out[0, h, :60001].cpu(), w[0, h, want])


@pytest.mark.parametrize("n,sequences,heads", [(300, 2, 3), (70000, 1, 2), (17, 3, 1)])
def test_evict_shared_weights(n, sequences, heads):
    """Weights that all heads, or all sequences and heads, have in common, without copies of them."""
    w = weights_of(9, sequences, 1, n, "ties")
    for shape in (w, w[:1]):
        f = Filled(23, [n] * sequences, heads, 64, 64, 64, F16)
        n_out, w_out, kept = api.evict_kv4(f.cache, f.table, ints([n] * sequences), shape.cuda().expand(sequences, heads, n), 13, recent=4)
        for b in range(sequences):
            for h in range(heads):
                mine = shape.expand(sequences, heads, n)[b, h]
                want = torch.cat([torch.sort(mine[:n - 4], descending=True, stable=True).indices[:9].sort().values, torch.arange(n - 4, n)])
                assert torch.equal(kept[b, h].cpu().long(), want) and same(w_out[b, h, :13].cpu(), mine[want]) and (w_out[b, h, 13:] == 0).all()


# ------------------------------------------------------------------------------------------------------------------- refusals

def test_refusals():
    f = Filled(22, [10, 20], 2, 64, 16, 64, BF16)
    q, k = torch.zeros(2, 4, 64, dtype=BF16, device="cuda"), torch.zeros(2, 2, 64, dtype=BF16, device="cuda")
    n, w = ints([10, 20]), torch.zeros(2, 2, 32, device="cuda")
    for bad in (lambda: api.attend_kv4(q.half(), f.cache, f.table, n), lambda: api.attend_kv4(q[:, :3], f.cache, f.table, n), lambda: api.attend_kv4(q[:1], f.cache, f.table, n),
                lambda: api.attend_kv4(q[..., :32], f.cache, f.table, n), lambda: api.attend_kv4(q, f.cache, f.table.long(), n), lambda: api.attend_kv4(q, f.cache, f.table, n.long()),
                lambda: api.attend_kv4(q, f.cache, f.table, n[:1]), lambda: api.attend_kv4(q, f.cache, f.table[0], n), lambda: api.attend_kv4(q, f.cache, f.table, n, ints([0, 2])),
                lambda: api.attend_kv4(q, f.cache, f.table, n, out=q), lambda: api.attend_kv4(q, f.cache, f.table, n, out=q[:1].clone()),
                lambda: api.attend_kv4(q, f.cache, f.table, n, weights=w[:1]), lambda: api.attend_kv4(q, f.cache, f.table, n, weights=w.double()),
                lambda: api.attend_kv4(q, f.cache, f.table, n, weights=w[:1, :1].expand(2, 2, 32)), lambda: api.attend_kv4(q.cpu(), f.cache, f.table, n),
                lambda: api.attend_kv4(q.clone().requires_grad_(), f.cache, f.table, n), lambda: api.attend_kv4(q, f.cache._replace(D=128), f.table, n),
                lambda: api.append_kv4(k, k[:1], f.cache, f.table, n), lambda: api.append_kv4(k[:, :1], k, f.cache, f.table, n), lambda: api.append_kv4(k, k.half(), f.cache, f.table, n),
                lambda: api.append_kv4(k, k.clone().requires_grad_(), f.cache, f.table, n), lambda: api.append_kv4(k, k, f.cache, f.table, n[:1]),
                lambda: api.read_kv4(f.cache, f.table, n, ints([0, 1, 2])), lambda: api.read_kv4(f.cache, f.table, n, ints([0, 1, 2]), total=-1),
                lambda: api.evict_kv4(f.cache, f.table, n, w, 0), lambda: api.evict_kv4(f.cache, f.table, n, w, 5, recent=6), lambda: api.evict_kv4(f.cache, f.table, n, w, 5, recent=-1),
                lambda: api.evict_kv4(f.cache, f.table, n, w, 17, into=f.table[:, :1]), lambda: api.evict_kv4(f.cache, f.table, n, w, 5, into=f.table[:1]),
                lambda: api.evict_kv4(f.cache, f.table, n, w, 5, into=f.table), lambda: api.evict_kv4(f.cache, f.table, n, torch.zeros(80, device="cuda").as_strided((2, 2, 32), (40, 8, 1)), 5),
                lambda: api.evict_kv4(f.cache, f.table, n, w[..., 0], 5), lambda: api.cache_kv4(4, 2, 80), lambda: api.cache_kv4(4, 2, 64, page=48), lambda: api.cache_kv4(4, 2, 64, group=48),
                lambda: api.cache_kv4(0, 2, 64), lambda: api.cache_kv4(4, 2, 64, dtype=torch.float32)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: api.attend_kv4(q, f.cache, f.table, n, scale=0.0), lambda: api.attend_kv4(q, f.cache, f.table, n, scale=-1.0), lambda: api.attend_kv4(q, f.cache, f.table, n, scale=math.nan),
                lambda: api.attend_kv4(torch.zeros(2 * 256 + 1, dtype=BF16, device="cuda")[1:].view(2, 4, 64), f.cache, f.table, n)):
        with pytest.raises(BitserialError):
            bad()
    with torch.no_grad():
        assert api.attend_kv4(q.clone().requires_grad_(), f.cache, f.table, n).shape == q.shape
