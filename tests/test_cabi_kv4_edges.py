"""Host-only checks of the entry points on keys and values of 4 bits: the largest sizes, refused before a device is touched."""
from test_cabi_kv4 import INVALID, OK, UNSUPPORTED, L, at, cache  # noqa: F401

MOST = 1 << 30


def test_more_entries_than_indices_reach(L, at):  # noqa: F811
    """Loops over entries and tokens step beyond the last one: sizes whose steps would pass 31 bits are refused."""
    def evict(width=4, page=64, into=None, iw=4, N=128, keep=10, work=at, size=1 << 62):
        return L.bs_kv4_evict(cache(at, page=page), at, width, width, into, iw, iw, 1, at, at, 1 << 40, 1 << 40, N, keep, 0, at, at, at, work, size, None)

    def attend(N):
        return L.bs_kv4_attend(at, 512, 128, 1, 2, cache(at), at, 4, 4, 1, at, None, 1.0, at, at, 1 << 40, 1 << 40, N, at, 1 << 62, None)

    def prompt(T=3, Tk=3):
        return L.bs_attend_prompt(at, 64, 64, T, 1, at, 64, 64, at, 64, 64, Tk, 1, 64, 2, 1, None, None, 1.0, 1, at, None)

    def append(T):
        return L.bs_kv4_append(at, 256, 128, at, 256, 128, T, cache(at), at, 4, 4, 1, at, at, None)

    def read(T):
        return L.bs_kv4_read(cache(at), at, 4, 4, 1, at, at, T, at, at, None)
    for n in (MOST + 1, 2 ** 31 - 1):
        assert evict(N=n) == evict(keep=n) == evict(N=n, into=at) == evict(keep=n, into=at) == UNSUPPORTED
        assert attend(n) == append(n) == read(n) == prompt(T=n) == prompt(Tk=n) == UNSUPPORTED
        assert L.bs_kv4_evict_workspace_bytes(cache(at), 1, n, 0) == 0
    assert L.bs_kv4_evict_workspace_bytes(cache(at), 1, MOST, 0) == MOST // 16 * 2 * 16 * (128 + 8)
    assert append(0) == read(0) == OK


def test_weights_that_share_memory(L, at):  # noqa: F811
    """Rows of weights that are added to may lie in any order, but not over one another."""
    def attend(sequence, head, B=3, N=100, T=None):
        return L.bs_kv4_attend(at, 512, 128, B if T is None else T, 4, cache(at), at, 4, 4, B, at, None if T is None else at, 1.0, at, at, sequence, head, N, at, 1 << 40, None)
    assert attend(0, 100) == attend(100, 100) == attend(199, 100) == attend(99, 400) == attend(100, 299) == attend(150, 150) == INVALID
    assert attend(200, 100, T=0) == attend(100, 300, T=0) == attend(0, 100, B=1, T=0) == OK
