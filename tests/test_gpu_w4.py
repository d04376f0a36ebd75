"""Grouped 4-bit weights on the GPU: quantiser, layout, the product with 16-bit activations and the mixture-of-experts layer, against their definitions in
64 bits (w4_reference.py).  Tolerances are the roundings': half a step of the output's type, and a step of the tensor cores' 32-bit sums for every
addition."""
import numpy as np
import pytest
import torch

import w4_reference as ref
from graph_launches import launches
from paper_2207_08820_b200 import api
from paper_2207_08820_b200._lib import BitserialError, lib

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
GUARD = 77.0


def weights(rng, O, K, group, dtype, zeros, lead=()):
    G = -(-K // group)
    codes = torch.from_numpy(rng.integers(0 if zeros else -8, 16 if zeros else 8, (*lead, O, K)).astype(np.int8))
    scales = torch.from_numpy(((rng.random((*lead, O, G)) + 0.5) * 0.2 / np.sqrt(K)).astype(np.float32)).to(dtype)
    z = torch.from_numpy(rng.integers(0, 16, (*lead, O, G)).astype(np.int8)) if zeros else None
    return codes, scales, z


def prepared(w, group):
    codes, scales, z = w
    return api.prepare_w4(codes.cuda(), scales.cuda(), None if z is None else z.cuda(), group=group)


def normal(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype)


def check_gemm(rng, M, O, K, group, dtype, zeros, bias):
    w = weights(rng, O, K, group, dtype, zeros)
    x, b = normal(rng, (M, K), dtype), normal(rng, (O,), dtype) if bias else None
    want, far = ref.gemm(x, ref.matrix(*w, group), b, dtype)
    # guard values around the output, its rows apart
    pitch = (O + 7) // 8 * 8 + 8
    room = torch.full((M + 2, pitch), GUARD, dtype=dtype, device="cuda")
    out = room[1:M + 1, :O]
    got = api.gemm_w4(x.cuda(), prepared(w, group), None if b is None else b.cuda(), out=out)
    api.bs_check_status()
    assert got.data_ptr() == out.data_ptr()
    assert ((out.cpu().double() - want).abs() <= far).all(), ((out.cpu().double() - want).abs() / far).max()
    room[1:M + 1, :O] = GUARD
    assert (room == GUARD).all(), "written beside the output"


# ------------------------------------------------------------------------------------------------------------------ quantiser

@pytest.mark.parametrize("source", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("O,K,group", [(1, 1, 32), (3, 40, 32), (17, 128, 128), (5, 131, 64), (9, 1000, 256), (33, 513, 384), (64, 264, 128), (7, 4096, 4096)])
def test_quantise(source, dtype, zeros, O, K, group):
    rng = np.random.default_rng(O * K + group)
    w = normal(rng, (O, K), source) * 0.05
    codes, scales, z = api.quantise_w4(w.cuda(), group, zeros=zeros, dtype=dtype)
    c, s, p = ref.quantise(w, group, zeros, dtype)
    assert np.array_equal(scales.double().cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), c)
    assert (z is None) == (not zeros) and (not zeros or np.array_equal(z.cpu().numpy(), p))
    if not zeros:       # half a step, and what the rounding of the scale (2^-9 of 7 steps at most, bf16) takes from the largest ones
        back = ref.matrix(codes.cpu(), scales.cpu(), None, group)
        step = scales.cpu().double()[:, torch.arange(K) // group]
        assert ((back - w.double()).abs() <= step * (0.5 + 7 * torch.finfo(dtype).eps)).all()


@pytest.mark.parametrize("zeros", [False, True])
def test_quantise_ties_and_extremes(zeros):
    """Quotients on ties and beside them by less than a float tells apart; groups of zeros, of values below the type, above it, infinities and NaN."""
    K = 32
    rows = []
    for s in (1.0, 0.75, 0.3203125):                 # the scale comes out as s: max / 7 (or the span / 15) is exact
        row = np.zeros(K, np.float64)
        row[0], row[1] = (15 * s, 0) if zeros else (7 * s, -7 * s)
        n = 6 if zeros else 3
        for i in range(10):
            t = np.float32((0.5 + i % n) * s)
            row[2 + 3 * i:5 + 3 * i] = [t, np.nextafter(t, np.float32(9)), np.nextafter(t, np.float32(-9))]
        rows.append(row)
    rows += [np.zeros(K), np.full(K, 1e-9), np.linspace(-1e30, 1e30, K), np.where(np.arange(K) == 3, np.inf, 1.0), np.where(np.arange(K) == 5, -np.inf, 1.0),
             np.where(np.arange(K) == 7, np.nan, 1.0), np.full(K, np.nan), np.full(K, -2.0)]
    w = torch.from_numpy(np.array(rows, np.float32))
    for dtype in (BF16, F16):
        for wide in (w, torch.cat([w, w[:, :1]], 1)[:, :K]):        # the second has rows of 33 floats: the other kernel
            src = wide.cuda() if wide.is_contiguous() else torch.cat([w, w[:, :1]], 1).cuda()[:, :K]
            codes, scales, z = api.quantise_w4(src, 32, zeros=zeros, dtype=dtype)
            c, s, p = ref.quantise(w, 32, zeros, dtype)
            assert np.array_equal(scales.double().cpu().numpy(), s)
            assert np.array_equal(codes.cpu().numpy(), c)
            assert not zeros or np.array_equal(z.cpu().numpy(), p)


def test_quantise_experts_and_defaults():
    rng = np.random.default_rng(5)
    w = normal(rng, (3, 10, 96), BF16)
    codes, scales, z = api.quantise_w4(w.cuda(), None)
    assert codes.shape == (3, 10, 96) and scales.shape == (3, 10, 1) and scales.dtype == BF16 and z is None
    one, s, _ = api.quantise_w4(w[1].cuda(), None)
    assert torch.equal(codes[1], one) and torch.equal(scales[1], s)
    assert api.quantise_w4(w.float().cuda())[1].dtype == BF16


# -------------------------------------------------------------------------------------------------------------------- product

@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("zeros,bias", [(False, False), (True, True)])
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("M,O,K", [(1, 1, 1), (1, 17, 129), (2, 16, 128), (3, 40, 100), (8, 33, 1000), (9, 64, 1152), (16, 100, 333), (17, 130, 260), (33, 31, 2050)])
def test_gemm_small(dtype, zeros, bias, group, M, O, K):
    check_gemm(np.random.default_rng(M * O + K + group), M, O, K, group, dtype, zeros, bias)


@pytest.mark.parametrize("M,O,K,group,dtype,zeros,bias", [
    (1, 4096, 4096, 128, BF16, False, False), (1, 6000, 1536, 384, F16, True, True), (8, 5000, 2304, 64, BF16, True, False),
    (31, 1383, 4611, 32, BF16, True, True), (64, 512, 4608, 128, F16, False, True), (65, 300, 640, 64, BF16, False, False),
    (127, 257, 2304, 128, BF16, True, False), (128, 128, 576, 128, F16, False, False), (129, 640, 1024, 1024, BF16, False, True),
    (200, 1024, 1000, 32, F16, True, True), (257, 384, 2056, 64, BF16, True, True), (300, 100, 264, 128, F16, False, False),
    (513, 2000, 512, 256, BF16, True, True), (65, 1100, 5003, 256, BF16, False, False),
    (128, 1024, 4200, 128, F16, True, True), (129, 700, 5760, 32, F16, False, True), (777, 130, 6000, 384, F16, False, True), (1000, 129, 1153, 128, F16, True, False)])
def test_gemm_larger(M, O, K, group, dtype, zeros, bias):
    check_gemm(np.random.default_rng(M + O + K), M, O, K, group, dtype, zeros, bias)


@pytest.mark.parametrize("M,O,K,group,dtype,zeros,bias", [
    (17, 8192, 5632, 128, BF16, False, True), (33, 4000, 5200, 64, F16, True, False), (64, 2047, 6600, 32, BF16, True, True),
    (65, 2000, 5003, 256, BF16, False, False), (128, 2048, 4200, 128, F16, True, True), (129, 1000, 5760, 32, F16, False, True),
    (200, 1000, 4096, 64, BF16, True, False), (300, 512, 4900, 128, BF16, True, True), (777, 200, 6000, 384, F16, False, True),
    (1000, 129, 5121, 1024, BF16, True, True), (2048, 100, 3333, 64, BF16, False, False), (4096, 1, 11000, 128, BF16, False, True),
    (4000, 333, 700, 32, BF16, True, True), (4096, 128, 1664, 128, F16, False, False), (9000, 2000, 100, 128, BF16, True, True)])
def test_gemm_many_rows(M, O, K, group, dtype, zeros, bias):
    """The kernel for many rows of x: one tile and many, cut and whole, all ways of groups."""
    check_gemm(np.random.default_rng(M + O + K), M, O, K, group, dtype, zeros, bias)


def test_gemm_cut_and_whole_tiles():
    """A reduction that is long enough to be cut asks for a workspace, a short one does not."""
    assert lib().bs_w4_gemm_workspace_bytes(200, 1000, 4096, 64, 4096) > 0
    assert lib().bs_w4_gemm_workspace_bytes(9000, 2000, 100, 128, 104) == 0


def test_gemm_whole_tiles_only():
    """As many tiles as multiprocessors, or twice as many: none is cut."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    check_gemm(np.random.default_rng(1), 128, 128 * sms, 264, 128, BF16, True, False)
    check_gemm(np.random.default_rng(2), 256, 128 * sms, 140, 64, F16, False, True)


@pytest.mark.parametrize("M", [1, 5, 20, 40, 150])
@pytest.mark.parametrize("pitch", [200, 203, 208])
def test_gemm_rows_apart(M, pitch):
    """Rows of x that are slices of wider ones, on and off 16-byte boundaries; what lies between them is NaN."""
    rng = np.random.default_rng(M + pitch)
    K, O, group = 197, 48, 64
    w = weights(rng, O, K, group, BF16, True)
    x = normal(rng, (M, K), BF16)
    wide = torch.full((M, pitch), float("nan"), dtype=BF16)
    wide[:, :K] = x
    want, far = ref.gemm(x, ref.matrix(*w, group), None, BF16)
    y = api.gemm_w4(wide.cuda()[:, :K], prepared(w, group))
    assert ((y.cpu().double() - want).abs() <= far).all()


def test_gemm_leading_dimensions_and_no_rows():
    rng = np.random.default_rng(1)
    w = prepared(weights(rng, 40, 72, 32, F16, False), 32)
    x = normal(rng, (2, 3, 72), F16).cuda()
    y = api.gemm_w4(x, w)
    assert y.shape == (2, 3, 40) and torch.equal(y.view(6, 40), api.gemm_w4(x.view(6, 72), w))
    assert torch.equal(api.gemm_w4(x[0, 0], w), api.gemm_w4(x[:1, 0], w)[0])
    assert api.gemm_w4(x[:0], w).shape == (0, 3, 40)


@pytest.mark.parametrize("M,K", [(5, 300), (150, 300), (4096, 1700)])
def test_gemm_special_values_stay_in_their_rows(M, K):
    rng = np.random.default_rng(M)
    w = weights(rng, 70, K, 32, BF16, True)
    x = normal(rng, (M, K), BF16)
    x[1, 7], x[3, K - 1] = float("inf"), float("nan")
    w[1][4, 2] = float("inf")
    want, far = ref.gemm(x, ref.matrix(*w, 32), None, BF16)
    y = api.gemm_w4(x.cuda(), prepared(w, 32)).cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(y), fine)
    assert ((y - want).abs()[fine] <= far[fine]).all()
    assert fine[0].sum() == 69 and not fine[1].any() and not fine[3].any()


@pytest.mark.parametrize("M,O,K", [(1, 2048, 2048), (16, 512, 1000), (64, 384, 2304), (300, 1000, 1152), (64, 2048, 6600), (300, 1000, 5000)])
def test_gemm_same_bits_every_time(M, O, K):
    rng = np.random.default_rng(M)
    w = prepared(weights(rng, O, K, 64, BF16, True), 64)
    x = normal(rng, (M, K), BF16).cuda()
    first = api.gemm_w4(x, w)
    for _ in range(20):
        assert torch.equal(api.gemm_w4(x, w), first)


@pytest.mark.parametrize("M,K", [(1, 512), (6, 515), (150, 512), (150, 515), (2048, 3304), (2048, 3301)])
def test_gemm_captured_beside_other_calls(M, K):
    """Two graphs of different products replayed in turn with eager calls between them: none reads what another keeps."""
    rng = np.random.default_rng(M)
    ws = [prepared(weights(rng, 200, K, 128, F16, False), 128) for _ in range(2)]
    xs = [normal(rng, (M, K), F16).cuda() for _ in range(2)]
    outs = [torch.empty(M, 200, dtype=F16, device="cuda") for _ in range(2)]
    api.gemm_w4(xs[0], ws[0])
    graphs = []
    for x, w, out in zip(xs, ws, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            api.gemm_w4(x, w, out=out)
        graphs.append(g)
    for _ in range(3):
        for x in xs:
            x.copy_(normal(rng, (M, K), F16))
        graphs[0].replay()
        eager = api.gemm_w4(xs[1], ws[0])
        graphs[1].replay()
        want = [api.gemm_w4(x, w) for x, w in zip(xs, ws)]
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
        assert torch.equal(eager, api.gemm_w4(xs[1], ws[0]))


@pytest.mark.parametrize("M,K", [(3, 1024), (3, 1023), (140, 1023), (1200, 3001)])
def test_gemm_on_another_stream(M, K):
    rng = np.random.default_rng(K)
    w = prepared(weights(rng, 300, K, 128, BF16, True), 128)
    xs = [normal(rng, (M, K), BF16).cuda() for _ in range(8)]
    want = [api.gemm_w4(x, w) for x in xs]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    got = [api.gemm_w4(x, w, stream=streams[i % 4]) for i, x in enumerate(xs)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_weights_prepared_and_used_at_once():
    """The product that follows the set-up in a stream reads what it wrote, also where the memory held other weights before."""
    rng = np.random.default_rng(8)
    sets = [weights(rng, 512, 1024, 128, BF16, False) for _ in range(4)]
    x = normal(rng, (2, 1024), BF16)
    on = [[t.cuda() for t in s[:2]] for s in sets]
    xd = x.cuda()
    for _ in range(5):
        got = [api.gemm_w4(xd, api.prepare_w4(c, s)) for c, s in on]
        for y, s in zip(got, sets):
            want, far = ref.gemm(x, ref.matrix(*s, 128), None, BF16)
            assert ((y.cpu().double() - want).abs() <= far).all()


# -------------------------------------------------------------------------------------------------------------------- experts

def moe_case(rng, T, E, H, I, gu, gd, dtype, zu, zd):
    gate, up = (weights(rng, I, H, gu, dtype, zu, (E,)) for _ in range(2))
    return normal(rng, (T, H), dtype), normal(rng, (E, H), dtype) / np.sqrt(H), gate, up, weights(rng, H, I, gd, dtype, zd, (E,))


def check_moe(x, router, gate, up, down, gu, gd, top_k, renormalise, xd=None):
    dtype = x.dtype
    want, far, experts, share = ref.moe(x, router, ref.matrix(*gate, gu), ref.matrix(*up, gu), ref.matrix(*down, gd), top_k, renormalise, dtype)
    y, e, s = api.moe_w4(x.cuda() if xd is None else xd, router.cuda(), prepared(gate, gu), prepared(up, gu), prepared(down, gd), top_k, renormalise=renormalise)
    assert torch.equal(e.cpu().long(), experts)
    assert ((s.cpu().double() - share).abs() <= share * 2.0 ** -19).all()
    assert ((y.cpu().double() - want).abs() <= far).all(), ((y.cpu().double() - want).abs() / far).max()
    return y


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("T,E,top_k,H,I,gu,gd,zu,zd,renormalise", [
    (1, 1, 1, 1, 1, 32, 32, False, False, True), (1, 4, 2, 128, 64, 128, 64, False, True, True), (3, 8, 8, 200, 48, 64, 32, True, False, False),
    (8, 16, 2, 256, 136, 128, 128, False, False, True), (9, 5, 3, 131, 77, 32, 32, True, True, False), (17, 33, 4, 264, 130, 64, 128, False, True, True),
    (37, 60, 4, 203, 141, 32, 64, True, True, False), (64, 128, 8, 160, 96, 128, 32, False, False, True), (65, 3, 2, 130, 150, 128, 128, True, False, True),
    (150, 2, 1, 96, 40, 32, 32, False, True, False), (20, 512, 32, 64, 33, 64, 32, True, True, True)])
def test_moe(dtype, T, E, top_k, H, I, gu, gd, zu, zd, renormalise):
    rng = np.random.default_rng(T * E + H)
    check_moe(*moe_case(rng, T, E, H, I, gu, gd, dtype, zu, zd), gu, gd, top_k, renormalise)


def test_moe_larger_reductions():
    rng = np.random.default_rng(3)
    check_moe(*moe_case(rng, 5, 6, 2304, 1160, 128, 128, BF16, False, False), 128, 128, 2, True)


@pytest.mark.parametrize("pitch", [72, 75])
def test_moe_rows_apart(pitch):
    rng = np.random.default_rng(pitch)
    case = moe_case(rng, 11, 6, 70, 50, 32, 32, BF16, True, False)
    wide = torch.full((11, pitch), float("nan"), dtype=BF16)
    wide[:, :70] = case[0]
    check_moe(*case, 32, 32, 3, True, xd=wide.cuda()[:, :70])


@pytest.mark.parametrize("T,E,top_k", [(64, 16, 8), (64, 128, 8), (64, 3, 3), (130, 7, 2), (8, 1, 1)])
def test_moe_writes_all_that_it_reads(T, E, top_k):
    """Experts with many tokens, whose work is cut in several parts; the workspace's memory holds NaN before every call."""
    rng = np.random.default_rng(T + E)
    x, router, gate, up, down = moe_case(rng, T, E, 256, 144, 128, 64, BF16, False, False)
    w = [prepared(p, q) for p, q in ((gate, 128), (up, 128), (down, 64))]
    want, far, _, _ = ref.moe(x, router, ref.matrix(*gate, 128), ref.matrix(*up, 128), ref.matrix(*down, 64), top_k, True, BF16)
    xd, rd = x.cuda(), router.cuda()
    for _ in range(10):
        poison = [torch.full((n << 10,), float("nan"), device="cuda") for n in (1, 8, 64, 128, 256, 512)]
        del poison
        y = api.moe_w4(xd, rd, *w, top_k)[0]
        assert ((y.cpu().double() - want).abs() <= far).all()


def test_moe_ties_and_equal_experts():
    """Equal logits: the lowest index first; all tokens to the same experts."""
    rng = np.random.default_rng(4)
    x, router, gate, up, down = moe_case(rng, 40, 9, 96, 64, 32, 32, F16, False, False)
    router[:] = router[0]
    check_moe(x, router, gate, up, down, 32, 32, 3, True)
    check_moe(torch.zeros_like(x), router, gate, up, down, 32, 32, 3, False)


def test_moe_special_values_stay_with_their_token():
    rng = np.random.default_rng(6)
    x, router, gate, up, down = moe_case(rng, 12, 6, 96, 64, 32, 32, BF16, False, False)
    w = [prepared(p, 32) for p in (gate, up, down)]
    good, _, _ = api.moe_w4(x.cuda(), router.cuda(), *w, 2)
    bad = x.clone()
    bad[3, 5], bad[7, 0] = float("nan"), float("inf")
    y, e, _ = api.moe_w4(bad.cuda(), router.cuda(), *w, 2)
    keep = [t for t in range(12) if t not in (3, 7)]
    assert torch.equal(y[keep], good[keep]) and not torch.isfinite(y[3]).any() and not torch.isfinite(y[7]).any()
    assert ((e >= 0) & (e < 6)).all() and (e[:, 0] != e[:, 1]).all()


def test_moe_hidden_values_beyond_fp16():
    """Hidden values far above what float16 holds, brought back by the last product."""
    rng = np.random.default_rng(7)
    x, router, gate, up, down = moe_case(rng, 3, 4, 128, 64, 128, 64, F16, False, False)
    gate[1].mul_(200), up[1].mul_(200), down[1].copy_(torch.full_like(down[1], 2.0 ** -14))
    y = check_moe(x, router, gate, up, down, 128, 64, 2, True)
    assert torch.isfinite(y).all()


def test_moe_same_bits_captured_and_on_streams():
    rng = np.random.default_rng(9)
    x, router, gate, up, down = moe_case(rng, 33, 16, 131, 90, 32, 32, BF16, True, True)
    w = [prepared(p, 32) for p in (gate, up, down)]
    xs = [x.cuda(), normal(rng, x.shape, BF16).cuda()]
    r = router.cuda()
    want = [[t.clone() for t in api.moe_w4(v, r, *w, 4)] for v in xs]
    graphs, outs = [], []
    for v in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(api.moe_w4(v, r, *w, 4))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(5):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        sided = [api.moe_w4(v, r, *w, 4, stream=s) for v, s in zip(xs, streams)]
        torch.cuda.synchronize()
        for got in (outs, sided):
            assert all(torch.equal(a, b) for o, q in zip(got, want) for a, b in zip(o, q))
    assert api.moe_w4(xs[0][:0], r, *w, 4)[0].shape == (0, 131)


# ---------------------------------------------------------------------------------------------------------------- run together

def test_layers_of_a_decoder_step():
    """As a program uses them: float weights quantised, prepared, a projection, experts on its outputs, a last projection."""
    rng = np.random.default_rng(11)
    H, I, E, T = 192, 128, 4, 3
    plain = {n: normal(rng, s, F32) / np.sqrt(s[-1]) for n, s in dict(a=(H, H), gate=(E, I, H), up=(E, I, H), down=(E, H, I), b=(50, H)).items()}
    q = {n: api.quantise_w4(w.cuda(), 64, zeros=n in ("a", "down")) for n, w in plain.items()}
    w = {n: api.prepare_w4(*v, group=64) for n, v in q.items()}
    m = {n: ref.matrix(*[None if t is None else t.cpu() for t in v], 64) for n, v in q.items()}
    x, router = normal(rng, (T, H), BF16), normal(rng, (E, H), BF16)
    h = api.gemm_w4(x.cuda(), w["a"])
    want, far = ref.gemm(x, m["a"], None, BF16)
    assert ((h.cpu().double() - want).abs() <= far).all()
    y, experts, _ = api.moe_w4(h, router.cuda(), w["gate"], w["up"], w["down"], 2)
    want, far, e, _ = ref.moe(h.cpu(), router, m["gate"], m["up"], m["down"], 2, True, BF16)
    assert torch.equal(experts.cpu().long(), e) and ((y.cpu().double() - want).abs() <= far).all()
    z = api.gemm_w4(y, w["b"])
    want, far = ref.gemm(y.cpu(), m["b"], None, BF16)
    assert ((z.cpu().double() - want).abs() <= far).all()


def test_refusals_on_the_device():
    rng = np.random.default_rng(2)
    w = prepared(weights(rng, 32, 64, 32, BF16, False), 32)
    x = normal(rng, (4, 64), BF16).cuda()
    for bad in (x.half(), x.float(), x[:, :63], x.cpu(), x.t().contiguous().t()):
        with pytest.raises(ValueError):
            api.gemm_w4(bad, w)
    with pytest.raises(ValueError):
        api.gemm_w4(x, w, bias=torch.zeros(31, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        api.gemm_w4(x, w, out=torch.empty(4, 33, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        api.gemm_w4(x, w._replace(O=64))
    with pytest.raises(ValueError):
        api.gemm_w4(x, w, out=x[:, :32])
    with pytest.raises(BitserialError):
        api.gemm_w4(torch.zeros(4 * 64 + 1, dtype=BF16, device="cuda")[1:].view(4, 64), w)      # off a 16-byte boundary
    with pytest.raises(BitserialError):
        api.quantise_w4(x, 48)
    with pytest.raises(ValueError):
        api.prepare_w4(torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, 3, dtype=BF16, device="cuda"), group=32)
    e = prepared(weights(rng, 32, 64, 32, BF16, False, (2,)), 32)
    d = prepared(weights(rng, 64, 32, 32, BF16, False, (2,)), 32)
    router = normal(rng, (2, 64), BF16).cuda()
    with pytest.raises(ValueError):
        api.moe_w4(x, router, e, e, d, 3)
    with pytest.raises(ValueError):
        api.moe_w4(x, router, e, e, e, 1)
    with pytest.raises(ValueError):
        api.gemm_w4(x, e)
    api.moe_w4(x, router, e, e, d, 2)
    api.bs_check_status()


def test_gemm_as_many_rows_as_are_taken():
    """The largest number of rows, with so little work in each that few-row tiles would be the fastest: more of them than a grid has."""
    rng = np.random.default_rng(12)
    w = weights(rng, 8, 16, 32, BF16, False)
    x = normal(rng, (1 << 20, 16), BF16)
    y = api.gemm_w4(x.cuda(), prepared(w, 32))
    api.bs_check_status()
    want, far = ref.gemm(x, ref.matrix(*w, 32), None, BF16)
    assert ((y.cpu().double() - want).abs() <= far).all()
    with pytest.raises(BitserialError):
        api.gemm_w4(torch.zeros((1 << 20) + 1, 16, dtype=BF16, device="cuda"), prepared(w, 32))


def test_one_token_without_a_batch():
    rng = np.random.default_rng(13)
    w = weights(rng, 40, 72, 32, F16, True)
    x = normal(rng, (72,), F16)
    y = api.gemm_w4(x.cuda(), prepared(w, 32))
    want, far = ref.gemm(x[None], ref.matrix(*w, 32), None, F16)
    assert y.shape == (40,) and ((y.cpu().double() - want[0]).abs() <= far[0]).all()
    xm, router, gate, up, down = moe_case(rng, 1, 5, 72, 40, 32, 32, F16, False, True)
    e = [prepared(p, 32) for p in (gate, up, down)]
    batch = api.moe_w4(xm.cuda(), router.cuda(), *e, 2)
    out = torch.empty(72, dtype=F16, device="cuda")
    single = api.moe_w4(xm[0].cuda(), router.cuda(), *e, 2, out=out)
    assert single[0].data_ptr() == out.data_ptr() and all(torch.equal(a, b[0]) for a, b in zip(single, batch))


def test_outputs_that_are_inputs_are_refused():
    rng = np.random.default_rng(14)
    w = prepared(weights(rng, 64, 64, 32, BF16, False), 32)
    x, bias = normal(rng, (1, 64), BF16).cuda(), normal(rng, (64,), BF16).cuda()
    e = prepared(weights(rng, 64, 64, 32, BF16, False, (2,)), 32)
    d = prepared(weights(rng, 64, 64, 32, BF16, False, (2,)), 32)
    router = normal(rng, (2, 64), BF16).cuda()
    with pytest.raises(ValueError):
        api.gemm_w4(x, w, bias, out=bias.view(1, 64))
    with pytest.raises(ValueError):
        api.gemm_w4(x, w, out=w.data[:128].view(BF16).view(1, 64))
    for out in (x, router[1:], e.data[:128].view(BF16).view(1, 64), d.data[:128].view(BF16).view(1, 64)):
        with pytest.raises(ValueError):
            api.moe_w4(x, router, e, e, d, 1, out=out)


@pytest.mark.parametrize("source", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("O,K,pitch,group", [(33, 513, 513, 128), (6, 1001, 1001, 256), (70, 259, 259, 32), (300, 31, 31, 64), (19, 264, 267, 128), (5, 384, 385, 32), (2, 129, 129, 128)])
def test_quantise_rows_off_wide_loads(source, zeros, O, K, pitch, group):
    """Rows of an odd number of columns or an odd distance apart; what lies between them is not read."""
    rng = np.random.default_rng(O + K)
    room = torch.full((O, pitch), float("inf"), dtype=source)
    room[:, :K] = normal(rng, (O, K), source) * 0.05
    codes, scales, z = api.quantise_w4(room.cuda()[:, :K], group, zeros=zeros, dtype=BF16)
    c, s, p = ref.quantise(room[:, :K], group, zeros, BF16)
    assert np.array_equal(scales.double().cpu().numpy(), s) and np.array_equal(codes.cpu().numpy(), c)
    assert not zeros or np.array_equal(z.cpu().numpy(), p)


def route(x, router, top_k, renormalise=True):
    """The choices and weights of a layer whose experts do not matter."""
    rng = np.random.default_rng(0)
    E, H = router.shape
    w = prepared(weights(rng, 16, H, 128, x.dtype, False, (E,)), 128)
    d = prepared(weights(rng, H, 16, 128, x.dtype, False, (E,)), 128)
    _, e, s = api.moe_w4(x.cuda(), router.cuda(), w, w, d, top_k, renormalise=renormalise)
    return e.cpu().long(), s.cpu().double()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("T,E,top_k,H", [(1, 2, 1, 64), (64, 16, 5, 64), (9, 40, 8, 71), (33, 128, 8, 264), (7, 512, 32, 64), (3, 200, 1, 1024)])
def test_moe_ties_between_different_sums(dtype, T, E, top_k, H):
    """Experts in pairs whose products are the same numbers in other columns, so that their logits are equal and 32-bit sums of them are not: the lower index
    first.  Every sum is exact in 64 bits: products are multiples of 2^-24 below 2^12, and there are fewer than 2^12 of them."""
    rng = np.random.default_rng(T + E)
    half = H // 2

    def wide(*shape):       # numbers of 8 bits, 2^-12 to 2^6
        return rng.integers(-128, 129, shape) * 2.0 ** rng.integers(-12, -1, shape)
    x = wide(T, H)
    x[:, half:2 * half] = x[:, :half]
    router = wide(E, H)
    swap = rng.random(half) < 0.5
    for e in range(1, E, 2):
        router[e] = router[e - 1]
        router[e, :half][swap], router[e, half:2 * half][swap] = router[e - 1, half:2 * half][swap], router[e - 1, :half][swap]
    x, router = torch.from_numpy(x).to(dtype), torch.from_numpy(router).to(dtype)
    logits = x.double() @ router.double().T
    assert E < 2 or torch.equal(logits[:, 0:E - 1:2], logits[:, 1::2])
    want = torch.sort(-logits, dim=-1, stable=True).indices[:, :top_k]
    got, _ = route(x, router, top_k)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("renormalise", [True, False])
def test_moe_logits_smaller_than_what_cancels(dtype, renormalise):
    """Products of 2^30 that cancel beside ones of 2^-2 and 2^-3, in one MMA's 16 products and in different ones: logits of 0.25, 0.125 and others near them."""
    E, H, T = 7, 128, 5
    x = torch.zeros(T, H, dtype=dtype)
    x[:, [0, 1, 2, 16, 32, 64, 100]] = 1
    x[:, 0] = x[:, 1] = x[:, 64] = 2.0 ** 15
    router = torch.zeros(E, H, dtype=dtype)
    router[0, 2] = 0.125
    router[1, [0, 1]] = torch.tensor([2.0 ** 15, -2.0 ** 15], dtype=dtype)
    router[1, 2] = 0.25
    router[2, [0, 64]] = torch.tensor([2.0 ** 15, -2.0 ** 15], dtype=dtype)
    router[2, 2] = 0.1875
    router[3, [1, 64]] = torch.tensor([-2.0 ** 15, 2.0 ** 15], dtype=dtype)
    router[3, [16, 100]] = 0.125
    router[4:, 2] = -1
    logits = x.double() @ router.double().T
    assert logits[0].tolist() == [0.125, 0.25, 0.1875, 0.25, -1, -1, -1]
    got, share = route(x, router, 4, renormalise)
    assert got.tolist() == [[1, 3, 2, 0]] * T
    p = torch.exp(logits)
    want = p.gather(1, got) / (p.gather(1, got) if renormalise else p).sum(1, keepdim=True)
    # expf of a difference rounded to 32 bits, its sum and the quotient: a few steps of a float
    assert ((share - want).abs() <= want * 2.0 ** -19).all()


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("E,O,K", [(260, 4099, 9), (3, 1 << 19, 8), (2, 1 << 20, 3)])
def test_quantise_stack_of_many_rows(zeros, E, O, K):
    """Experts that together have more rows than one matrix may have."""
    rng = np.random.default_rng(E)
    w = normal(rng, (E, O, K), BF16)
    codes, scales, z = api.quantise_w4(w.cuda(), 32, zeros=zeros)
    c, s, p = ref.quantise(w.view(E * O, K), 32, zeros, BF16)
    assert codes.shape == w.shape and scales.shape == (E, O, 1)
    assert np.array_equal(scales.view(E * O, 1).double().cpu().numpy(), s) and np.array_equal(codes.view(E * O, K).cpu().numpy(), c)
    assert not zeros or np.array_equal(z.view(E * O, 1).cpu().numpy(), p)
    api.prepare_w4(codes, scales, z, group=32)
    api.bs_check_status()


def test_quantise_matrix_of_too_many_rows():
    for shape in (((1 << 20) + 1, 2), (1, (1 << 20) + 1, 2)):
        with pytest.raises(BitserialError):
            api.quantise_w4(torch.zeros(shape, dtype=BF16, device="cuda"), 32)


@pytest.mark.parametrize("M,O,K", [(3, 40, 72), (40, 200, 1000), (300, 1000, 4904), (2, 8, 8)])
@pytest.mark.parametrize("first", ["x", "out"])
def test_gemm_output_beside_its_input(M, O, K, first):
    """x and the output are columns of one buffer; a column in common, in the same row or in the next one, is refused."""
    rng = np.random.default_rng(M)
    w = weights(rng, O, K, 128, BF16, False)
    x = normal(rng, (M, K), BF16)
    want, far = ref.gemm(x, ref.matrix(*w, 128), None, BF16)
    wp = prepared(w, 128)
    pitch = K + O + 8
    room = torch.full((M, pitch), GUARD, dtype=BF16, device="cuda")
    x0, o0 = (0, K) if first == "x" else (O + 8, 0)
    room[:, x0:x0 + K] = x.cuda()
    out = room[:, o0:o0 + O]
    api.gemm_w4(room[:, x0:x0 + K], wp, out=out)
    assert ((out.cpu().double() - want).abs() <= far).all()
    assert torch.equal(room[:, x0:x0 + K].cpu(), x)
    room[:, x0:x0 + K], room[:, o0:o0 + O] = GUARD, GUARD
    assert (room == GUARD).all()
    flat = torch.zeros(M * pitch + 64, dtype=BF16, device="cuda")
    for step, at in ((K + O, K - 8), (K + O, K + 8), (K + O - 8, K)):       # into x's row; into the next one
        with pytest.raises(ValueError):
            api.gemm_w4(flat.as_strided((M, K), (step, 1), 0), wp, out=flat.as_strided((M, O), (step, 1), at))
    with pytest.raises(ValueError):
        api.gemm_w4(flat.as_strided((M, K), (K + O, 1), O - 8), wp, out=flat.as_strided((M, O), (K + O, 1), 0))


@pytest.mark.parametrize("T,E,top_k,H,I,items", [(64, 4, 4, 2048, 768, 512), (64, 8, 8, 512, 512, 512), (130, 4, 1, 2048, 768, 192)])
def test_moe_few_experts_with_many_slots(T, E, top_k, H, I, items):
    """An expert's slots are cut in jobs of eight: both products get a CTA for every place of the GPU, as there are jobs enough, or one for every item.  The second
    product's items: 32, 64 and at most 4 + 64 / 8 jobs, of 16, 8 and 16 times 32 rows by teams of two (768 columns) or four warps (512)."""
    rng = np.random.default_rng(T + E + H)
    x, router, gate, up, down = moe_case(rng, T, E, H, I, 128, 128, BF16, False, False)
    w = [prepared(p, 128) for p in (gate, up, down)]
    xd, rd = x.cuda(), router.cuda()
    grids = dict(launches(lambda: api.moe_w4(xd, rd, *w, top_k)))
    places = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    for name, want in (("w4_moe_gate_kernel", places), ("w4_moe_down_kernel", min(places, items))):
        assert [grid[0] for kernel, grid in grids.items() if name in kernel] == [want]
    some = x[:9]        # the definition, of some of the tokens
    want, far, _, _ = ref.moe(some, router, ref.matrix(*gate, 128), ref.matrix(*up, 128), ref.matrix(*down, 128), top_k, True, BF16)
    y = api.moe_w4(xd, rd, *w, top_k)[0][:9]
    assert ((y.cpu().double() - want).abs() <= far).all()


def product_kernel(M, O, K, group, dtype, zeros, bias):
    """Which of the two kernels a product launches."""
    w = prepared(weights(np.random.default_rng(0), O, K, group, dtype, zeros), group)
    x, b = torch.zeros(M, K, dtype=dtype, device="cuda"), torch.zeros(O, dtype=dtype, device="cuda") if bias else None
    names = [name for name, _ in launches(lambda: api.gemm_w4(x, w, b))]
    return [kernel for kernel in ("w4_gemm_kernel", "w4_mma_kernel") if any(kernel in name for name in names)]


MANY_ROWS = [
    (17, 8192, 5632, 128, BF16, False, True), (33, 4000, 5200, 64, F16, True, False), (64, 2047, 6600, 32, BF16, True, True),
    (65, 2000, 5003, 256, BF16, False, False), (128, 2048, 4200, 128, F16, True, True), (129, 1000, 5760, 32, F16, False, True),
    (200, 1000, 4096, 64, BF16, True, False), (300, 512, 4900, 128, BF16, True, True), (777, 200, 6000, 384, F16, False, True),
    (1000, 129, 5121, 1024, BF16, True, True), (2048, 100, 3333, 64, BF16, False, False), (4000, 333, 700, 32, BF16, True, True),
    (4096, 128, 1664, 128, F16, False, False), (9000, 2000, 100, 128, BF16, True, True)]
FEW_OUTPUTS = [(4096, 20, 11000, 128, BF16, False, True), (4096, 17, 11001, 128, F16, True, False), (1 << 20, 1, 16, 32, BF16, True, True)]


@pytest.mark.parametrize("case", MANY_ROWS + FEW_OUTPUTS, ids=str)
def test_gemm_products_of_the_kernel_for_many_rows(case):
    assert product_kernel(*case) == ["w4_mma_kernel"]


@pytest.mark.parametrize("case", [(1, 24576, 8192, 128, BF16, False, False), (16, 4096, 4096, 128, BF16, False, False), (33, 31, 2050, 32, F16, True, True), (4096, 1, 11000, 128, BF16, False, True)], ids=str)
def test_gemm_products_of_the_kernel_for_few_rows(case):
    """Up to 16 rows, and more where there is little work in each."""
    assert product_kernel(*case) == ["w4_gemm_kernel"]


@pytest.mark.parametrize("M,O,K,group,dtype,zeros,bias", FEW_OUTPUTS)
def test_gemm_many_rows_of_few_outputs(M, O, K, group, dtype, zeros, bias):
    check_gemm(np.random.default_rng(O + K), M, O, K, group, dtype, zeros, bias)


@pytest.mark.parametrize("what", ["quantise", "prepare", "gemm", "moe"])
def test_inputs_let_go_of_before_another_stream_has_read_them(what):
    """A call on a stream that is still busy, its inputs dropped at once and their memory asked for again on the current stream."""
    rng = np.random.default_rng(15)
    H, T = 256, 64
    plain = normal(rng, (H, H), BF16)
    codes, scales, _ = weights(rng, H, H, 128, BF16, False)
    w = prepared((codes, scales, None), 128)
    e = [prepared(weights(rng, H, H, 128, BF16, False, (4,)), 128) for _ in range(3)]
    x, router, bias = normal(rng, (T, H), BF16), normal(rng, (4, H), BF16), normal(rng, (H,), BF16)
    calls = dict(quantise=((plain,), lambda w, **k: api.quantise_w4(w, **k)[:2]),
                 prepare=((codes, scales), lambda c, s, **k: (api.prepare_w4(c, s, **k).data,)),
                 gemm=((x, bias), lambda x, b, **k: (api.gemm_w4(x, w, b, **k),)),
                 moe=((x, router), lambda x, r, **k: api.moe_w4(x, r, *e, 2, **k)))
    inputs, call = calls[what]
    want = call(*[t.cuda() for t in inputs])
    side = torch.cuda.Stream()
    for t in inputs:        # a kernel's first launch waits for all streams
        torch.full(t.shape, 3, dtype=t.dtype, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    given = [t.cuda() for t in inputs]
    places = {t.data_ptr() for t in given}
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)      # 0.2 s
    got = call(*given, stream=side)
    del given
    junk = [torch.full(t.shape, 3, dtype=t.dtype, device="cuda") for t in inputs for _ in range(3)]
    assert not side.query(), "the stream was to be busy until here"
    assert not places & {t.data_ptr() for t in junk}
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_with_the_stream_named():
    """The capturing stream given by name, with an input that lives in the capture alone."""
    rng = np.random.default_rng(16)
    w = prepared(weights(rng, 100, 136, 64, F16, True), 64)
    x = normal(rng, (5, 136), F16).cuda()
    out = torch.empty(5, 100, dtype=F16, device="cuda")
    api.gemm_w4(x + x, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.gemm_w4(x + x, w, out=out, stream=torch.cuda.current_stream())
    for _ in range(2):
        x.copy_(normal(rng, (5, 136), F16))
        graph.replay()
        assert torch.equal(out, api.gemm_w4(x + x, w))
