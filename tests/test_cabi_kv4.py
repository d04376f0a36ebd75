"""Host-only checks of the entry points on keys and values of 4 bits: sizes, and refusals before a device is touched."""
import ctypes

import pytest

OK, INVALID, UNSUPPORTED, ALIGN = 0, 1, 2, 3
F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    from paper_2207_08820_b200 import build
    build.build()
    from paper_2207_08820_b200 import _lib
    return _lib.lib()


@pytest.fixture(scope="module")
def at():
    buf = (ctypes.c_char * 8192)()
    yield (ctypes.addressof(buf) + 255) & ~255      # never dereferenced: validation fails first


def cache(at, data=True, pages=4, heads=2, D=128, page=64, group=128, type=BF16):
    from paper_2207_08820_b200._lib import KV4CacheDesc
    return ctypes.byref(KV4CacheDesc(at if data is True else data, pages, heads, D, page, group, type))


BAD_LAYOUTS = [dict(D=80), dict(D=256), dict(group=48), dict(group=96), dict(page=8), dict(page=48), dict(page=2048), dict(heads=65536)]
BAD_CACHES = [dict(data=None), dict(pages=0), dict(heads=0), dict(D=0), dict(page=0), dict(group=0), dict(type=F32), dict(type=7)]


def test_sizes(L):
    assert L.bs_kv4_page_bytes(1, 128, 16, 128) == 16 * (128 + 8)
    assert L.bs_kv4_page_bytes(8, 128, 64, 32) == 8 * 64 * (128 + 32)
    assert L.bs_kv4_page_bytes(3, 96, 32, 96) == 3 * 32 * (96 + 8)
    assert L.bs_kv4_page_bytes(3, 64, 1024, 32) == 3 * 1024 * (64 + 16)
    for heads, D, page, group in ((0, 128, 64, 128), (1, 80, 64, 80), (1, 128, 8, 128), (1, 128, 24, 128), (1, 128, 2048, 128), (1, 128, 64, 48), (1, 96, 64, 64), (1, 128, 64, 0), (70000, 64, 64, 64)):
        assert L.bs_kv4_page_bytes(heads, D, page, group) == 0


def test_evict_workspace(L, at):
    assert L.bs_kv4_evict_workspace_bytes(cache(at), 3, 17, 0) == 3 * 2 * 2 * 16 * (128 + 8)
    assert L.bs_kv4_evict_workspace_bytes(cache(at), 3, 17, 1) == 0
    assert L.bs_kv4_evict_workspace_bytes(cache(at, D=80), 3, 17, 0) == L.bs_kv4_evict_workspace_bytes(cache(at), 0, 17, 0) == L.bs_kv4_evict_workspace_bytes(cache(at), 3, 0, 0) == 0


def test_append_and_read_refuse(L, at):
    def append(k=at, kt=256, kh=128, v=at, vt=256, vh=128, T=2, c=None, table=at, pitch=4, width=4, B=2, first=at, starts=None):
        return L.bs_kv4_append(k, kt, kh, v, vt, vh, T, c or cache(at), table, pitch, width, B, first, starts, None)

    def read(c=None, table=at, pitch=4, width=4, B=2, first=at, starts=None, T=2, k=at, v=at):
        return L.bs_kv4_read(c or cache(at), table, pitch, width, B, first, starts, T, k, v, None)
    for f in (append, read):
        assert f(k=None) == f(v=None) == f(table=None) == f(first=None) == f(T=-1) == f(T=3) == f(B=0) == f(width=0) == f(pitch=3) == INVALID
        assert f(k=at + 2) == f(v=at + 8) == f(c=cache(at, data=at + 4)) == ALIGN
        assert all(f(c=cache(at, **bad)) == INVALID for bad in BAD_CACHES)
        assert all(f(c=cache(at, **bad)) == UNSUPPORTED for bad in BAD_LAYOUTS)
        assert f(T=0, starts=at) == OK
    assert append(kt=-8) == append(vh=-8) == INVALID
    assert append(kt=257) == append(kh=4) == append(vt=1) == append(vh=9) == ALIGN


def test_attend_refuses(L, at):
    def attend(q=at, qt=512, qh=128, T=2, heads=4, c=None, table=at, pitch=4, width=4, B=2, lengths=at, starts=None, scale=1.0, out=at, w=None, ws=256, wh=128, N=128, work=at, size=1 << 30):
        return L.bs_kv4_attend(q, qt, qh, T, heads, c or cache(at), table, pitch, width, B, lengths, starts, scale, out, w, ws, wh, N, work, size, None)
    assert attend(q=None) == attend(table=None) == attend(lengths=None) == attend(out=None) == INVALID
    assert attend(T=-1) == attend(T=3) == attend(heads=3) == attend(heads=0) == attend(B=0) == attend(width=0) == attend(pitch=3) == attend(qt=-8) == INVALID
    assert attend(scale=3e38) == INVALID         # times log2(e) it is no number of binary32
    assert attend(scale=0.0) == attend(scale=-1.0) == attend(scale=float("inf")) == attend(scale=float("nan")) == INVALID
    assert attend(w=at, N=0) == attend(w=at, wh=127) == attend(w=at, ws=-1) == INVALID
    assert attend(q=at + 2) == attend(out=at + 4) == attend(work=at + 8) == attend(qt=1) == attend(qh=4) == ALIGN
    assert all(attend(c=cache(at, **bad)) == INVALID for bad in BAD_CACHES)
    assert all(attend(c=cache(at, **bad)) in (INVALID, UNSUPPORTED) for bad in BAD_LAYOUTS)
    assert attend(c=cache(at, D=80)) == UNSUPPORTED
    assert attend(T=0, starts=at) == OK


def test_evict_refuses(L, at):
    def evict(c=None, table=at, pitch=4, width=4, into=None, ip=4, iw=4, B=2, lengths=at, w=at, ws=256, wh=128, N=128, keep=10, recent=3, n=at, wo=at, kept=at, work=at, size=1 << 30):
        return L.bs_kv4_evict(c or cache(at), table, pitch, width, into, ip, iw, B, lengths, w, ws, wh, N, keep, recent, n, wo, kept, work, size, None)
    assert evict(table=None) == evict(lengths=None) == evict(w=None) == evict(n=None) == evict(wo=None) == evict(kept=None) == INVALID
    assert evict(width=0) == evict(pitch=3) == evict(B=0) == evict(N=0) == evict(keep=0) == evict(recent=-1) == evict(recent=11) == evict(wh=127) == evict(wh=-128) == evict(ws=-1) == INVALID
    assert evict(work=None) == evict(size=2 * 2 * 16 * 136 - 1) == INVALID
    assert evict(into=at, iw=0) == evict(into=at, ip=3) == evict(into=at, iw=1, keep=65) == INVALID
    assert evict(work=at + 8) == evict(c=cache(at, data=at + 4)) == ALIGN
    assert all(evict(c=cache(at, **bad)) == INVALID for bad in BAD_CACHES)
    assert all(evict(c=cache(at, **bad)) == UNSUPPORTED for bad in BAD_LAYOUTS)
    assert evict(B=65536) == UNSUPPORTED


def test_prompt_refuses(L, at):
    def prompt(q=at, qt=256, qh=64, T=3, heads=4, k=at, kt=128, kh=64, v=at, vt=128, vh=64, Tk=3, kv=2, D=64, type=BF16, B=1, s=at, sk=at, scale=1.0, out=at):
        return L.bs_attend_prompt(q, qt, qh, T, heads, k, kt, kh, v, vt, vh, Tk, kv, D, type, B, s, sk, scale, 1, out, None)
    assert prompt(q=None) == prompt(k=None) == prompt(v=None) == prompt(out=None) == INVALID
    assert prompt(T=-1) == prompt(Tk=-1) == prompt(heads=3) == prompt(heads=0) == prompt(kv=0) == prompt(D=0) == prompt(B=0) == INVALID
    assert prompt(scale=3e38) == INVALID
    assert prompt(type=F32) == prompt(type=9) == prompt(scale=0.0) == prompt(scale=-2.0) == prompt(scale=float("inf")) == prompt(scale=float("nan")) == INVALID
    assert prompt(s=None) == prompt(sk=None) == prompt(s=None, sk=None, B=2) == prompt(qt=-8) == prompt(kh=-8) == prompt(vt=-8) == INVALID
    assert prompt(D=136) == prompt(D=60) == prompt(heads=258) == UNSUPPORTED
    assert prompt(q=at + 2) == prompt(k=at + 8) == prompt(v=at + 4) == prompt(out=at + 2) == prompt(qt=257) == prompt(kh=4) == prompt(vh=2) == ALIGN
    assert prompt(T=0) == OK
