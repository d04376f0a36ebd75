// Eviction from a cache of 4-bit keys and values: every head keeps its newest entries and, of the others, those that got most attention, in their order.
//
// A CTA, or a cluster of them where the entries are many, takes a head of a sequence.  The least weight that stays is found by its digits, 11, 11 and 10 bits from
// the top of a key whose order as a whole number is that of the weights: each CTA counts its part of the entries by digit in shared memory, adds a part of
// the digits up over the cluster and hands the sums to all.  Entries above it stay, of those equal to it the first ones.  A second pass over the entries writes the
// indices, ranked by sums over warps and CTAs.  What stays is then moved by a kernel over all heads and sequences: into other pages at once, into their own
// through a copy, since what one CTA writes another may still have to read.
//
// Sequences with entries or places that are not there, on pages that the cache does not have, go a way of their own behind this one: one CTA a head, the least weight bit
// by bit.  Looking for such pages takes half a microsecond to one (4096 entries to 2048 and read back: 17.4 us without, 18.0 with it).
//
// 16 sequences of up to 32768 entries and 8 heads cut to 8191: 33 us to select (four weights a thread and turn; with one 52), bound by loads and atomics, 55 to move at
// 4 TB/s.  16 sequences of 32768, bf16, one group a head: 120 us into other pages, 181 in place, where every byte moves twice; with weights that are all the same 112 into
// other pages.  4096 entries to 2048: 12.6 us with the launches, 15.2 in place.
#include "kv4.h"
#include "mma_kernel.cuh"
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int THREADS = 1024, BINS = 2048, MOST = 8;            // MOST: CTAs of a cluster

struct Evict {
    Kv4 l;
    Kv4Table from, into;
    const int32_t* lengths;
    const float* weights;
    long long w_sequence, w_head;
    int N, keep, recent;
    int inside;                 // into the sequences' own pages
    int32_t* lengths_out;       // [B]
    float* weights_out;         // [B][H][N]
    int32_t* kept;              // [B][H][keep]
    unsigned char* copy;        // [B][H][ceil(keep / 16)] tiles, for moves within a sequence's own pages
};

__device__ __forceinline__ uint32_t key_of(float w)
{
    if (w != w) return 0xffffffffu;         // NaN comes first
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint32_t mapped(const void* p, int rank)
{
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ uint32_t remote(const void* p, int rank)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(mapped(p, rank)));
    return v;
}
__device__ __forceinline__ int entries_of(const Evict& a, const int32_t* lengths, int b)
{
    const long long room = min(static_cast<long long>(a.from.width) * a.l.page, static_cast<long long>(a.N));
    const int n = lengths[b];
    return n < 0 ? 0 : n > room ? static_cast<int>(room) : n;
}
__device__ __forceinline__ uint32_t up_to_lane(uint32_t s)
{
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, s, d);
        if ((threadIdx.x & 31) >= d) s += u;
    }
    return s;
}
// Four neighbouring weights, of those below `to`; others as keys that come last.
__device__ __forceinline__ void load4(const float* w, int i, int to, bool vectors, float (&v)[4])
{
    if (vectors && i + 4 <= to) {
        const float4 x = *reinterpret_cast<const float4*>(w + i);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = i + j < to ? w[i + j] : 0.f;
    }
}
// Sum over the threads before this one; all: over all of them.  32 warps.
__device__ __forceinline__ uint32_t before_me(uint32_t v, uint32_t* sums, uint32_t& all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t s = up_to_lane(v);
    if (lane == 31) sums[warp] = s;
    __syncthreads();
    const uint32_t w = up_to_lane(sums[lane]);
    all = __shfl_sync(0xffffffffu, w, 31);
    const uint32_t front = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    __syncthreads();
    return (warp ? front : 0u) + s - v;
}

// A head's entries and places, 0 to `from` and to `into` (some of them not there): what stays takes the places that are there, in order.  By a CTA, for few sequences, so
// without haste: every count is one over the pages, or over the weights for each of their bits.
__device__ __forceinline__ void select_around(const Evict& a, const Kv4Table& from, const Kv4Table& into, int b, int n, const float* w, int32_t* kept, float* out, int32_t* length, uint32_t* sums)
{
    const int th = threadIdx.x;
    auto count = [&](const Kv4Table& t, int lo, int hi) {           // of those in lo .. hi - 1 that are there
        uint32_t mine = 0, all;
        for (long long p = (lo >> a.l.log_page) + th; p << a.l.log_page < hi; p += THREADS) {
            const long long first = p << a.l.log_page, last = first + a.l.page;
            if (kv4_page_of(a.l, t, b, first) >= 0) mine += static_cast<uint32_t>(min(last, static_cast<long long>(hi)) - max(first, static_cast<long long>(lo)));
        }
        before_me(mine, sums, all);
        return static_cast<int>(all);
    };
    const int places = static_cast<int>(min(static_cast<long long>(into.width) * a.l.page, static_cast<long long>(min(a.keep, a.N))));
    const int entries = count(from, 0, n), room = count(into, 0, places), stay = min(entries, room), newest = entries > room ? min(a.recent, stay) : stay;
    int old = 0;
    if (entries > room) {           // the newest ones begin where so many follow
        int hi = n;
        while (hi - old > 1) {
            const int mid = old + ((hi - old) >> 1);
            if (count(from, mid, n) >= newest) old = mid;
            else hi = mid;
        }
        if (newest == 0) old = n;
    }
    const uint32_t need = stay - newest;
    auto is_there = [&](const Kv4Table& t, int i, int end) { return i < end && kv4_page_of(a.l, t, b, i) >= 0; };
    auto above = [&](uint32_t key) {            // how many of the older ones have it or a greater one
        uint32_t mine = 0, all;
        for (long long i = th; i < old; i += THREADS) mine += is_there(from, static_cast<int>(i), old) && key_of(w[i]) >= key;
        before_me(mine, sums, all);
        return all;
    };
    uint32_t least = 0;             // the least key that stays
    for (int bit = 31; bit >= 0 && need > 0; --bit)
        if (above(least | 1u << bit) >= need) least |= 1u << bit;
    const uint32_t left = need == 0 ? 0u : need - (least == 0xffffffffu ? 0u : above(least + 1));        // of those equal to it
    uint32_t rank = 0, equal = 0;
    for (long long i0 = 0; i0 < n; i0 += THREADS) {
        const int i = static_cast<int>(i0 + th < n ? i0 + th : n);
        const bool there = is_there(from, i, n);
        const uint32_t key = there && i < old ? key_of(w[i]) : 0u, same = need > 0 && there && i < old && key == least;
        uint32_t all_same, all;
        const uint32_t mine = equal + before_me(same, sums, all_same);
        const uint32_t stays = there && (i >= old || (need > 0 && key > least) || (same && mine < left));
        const uint32_t at = rank + before_me(stays, sums, all);
        if (stays && at < static_cast<uint32_t>(stay)) kept[at] = i;            // the latter but for weights that change meanwhile
        rank += all;
        equal += all_same;
    }
    // from ranks to places, from the last ones on: a place is not before its rank
    uint32_t left_places = room;
    if (th == 0 && stay == 0 && length) *length = 0;
    for (long long r0 = (static_cast<long long>(a.keep) - 1) / THREADS * THREADS; r0 >= 0; r0 -= THREADS) {
        const long long r = r0 + th;
        const uint32_t there = r < places && is_there(into, static_cast<int>(r), places);
        uint32_t all;
        const uint32_t mine = before_me(there, sums, all), at = left_places - all + mine;
        const int i = there && at < static_cast<uint32_t>(stay) ? kept[at] : -1;
        __syncthreads();
        if (r < a.keep) kept[r] = i;
        if (r < places) out[r] = i >= 0 ? w[i] : 0.f;
        if (there && at + 1 == static_cast<uint32_t>(stay) && length) *length = static_cast<int>(r) + 1;
        left_places -= all;
    }
    for (long long r = places + th; r < a.N; r += THREADS) out[r] = 0.f;
}

// CTAS: of the cluster.
template <int CTAS>
__global__ void __launch_bounds__(THREADS, 2) kv4_select_kernel(const __grid_constant__ Evict a)
{
    __shared__ uint32_t bins[3][BINS], sums[THREADS / 32], found[2], mine[2];
    __shared__ uint32_t digits[CTAS == 1 ? 1 : BINS];           // sums over the cluster
    auto sync = [] { if (CTAS == 1) __syncthreads(); else mm_cluster_sync(); };
    dependent_begin(a.kept);
    const int rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z, th = threadIdx.x;
    const int n = entries_of(a, behind_wait<int32_t>(a.lengths), b);
    const float* w = behind_wait<float>(a.weights) + b * a.w_sequence + h * a.w_head;
    const long long head = static_cast<long long>(b) * a.l.H + h;
    int32_t* kept = a.kept + head * a.keep;
    float* out = a.weights_out + head * a.N;
    const int stay = min(n, a.keep), old = n > a.keep ? n - a.recent : 0, need = n > a.keep ? a.keep - a.recent : 0;
    // the CTA's part, in fours
    const int from = static_cast<int>(static_cast<long long>(old) * rank / CTAS) & ~3, to = rank + 1 == CTAS ? old : static_cast<int>(static_cast<long long>(old) * (rank + 1) / CTAS) & ~3;
    const bool vectors = (reinterpret_cast<uintptr_t>(w) & 15) == 0;
    // whether an entry, or a place of one that stays, is not there (sequences that stay in place do not care): asked here, where other loads cover it, and answered last
    Kv4Table own = a.from, other = a.into;
    own.pages = behind_wait<int32_t>(a.from.pages);
    other.pages = behind_wait<int32_t>(a.into.pages);
    bool missing = false;
    if (n > a.keep || !a.inside) {
        for (int p = th; p << a.l.log_page < n; p += THREADS) missing |= kv4_page_of(a.l, own, b, p << a.l.log_page) < 0;
        for (int p = th; !a.inside && p << a.l.log_page < stay; p += THREADS) missing |= kv4_page_of(a.l, other, b, p << a.l.log_page) < 0;
    }
    if (need > 0) {
        for (int i = th; i < 3 * BINS; i += THREADS) (&bins[0][0])[i] = 0;
        __syncthreads();
        uint32_t prefix = 0, left = need;           // digits found; how many entries of that prefix stay
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, wide = pass == 2 ? 10 : 11;
#pragma unroll 4
            for (int i = from + 4 * th; i < to; i += 4 * THREADS) {
                float v[4];
                load4(w, i, to, vectors, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t k = key_of(v[j]);
                    if (i + j < to && (pass == 0 || k >> (shift + wide) == prefix)) atomicAdd(&bins[pass][k >> shift & ((1u << wide) - 1)], 1u);
                }
            }
            sync();
            const uint32_t* count = bins[pass];
            if (CTAS > 1) {
                constexpr int SLICE = BINS / CTAS;
                for (int i = th; i < SLICE; i += THREADS) {
                    const int digit = rank * SLICE + i;
                    uint32_t v[CTAS], sum = 0;
#pragma unroll
                    for (int c = 0; c < CTAS; ++c) v[c] = remote(&bins[pass][digit], c);
#pragma unroll
                    for (int c = 0; c < CTAS; ++c) sum += v[c];
#pragma unroll
                    for (int c = 0; c < CTAS; ++c) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapped(&digits[digit], c)), "r"(sum) : "memory");
                }
                sync();
                count = digits;
            }
            // two digits a thread, from the top down
            const int top = BINS - 1 - 2 * th;
            const uint32_t c0 = count[top], c1 = count[top - 1];
            uint32_t all, above = before_me(c0 + c1, sums, all);
            if (above < left && left <= above + c0) { found[0] = top; found[1] = left - above; }
            above += c0;
            if (above < left && left <= above + c1) { found[0] = top - 1; found[1] = left - above; }
            __syncthreads();
            prefix = prefix << wide | found[0];
            left = found[1];
            __syncthreads();
        }
        // `left` entries equal to `prefix` stay, and all above it
        uint32_t at_more = 0, at_equal = 0;
        if (CTAS > 1) {
            uint32_t more = 0, equal = 0;
#pragma unroll 4
            for (int i = from + 4 * th; i < to; i += 4 * THREADS) {
                float v[4];
                load4(w, i, to, vectors, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t k = key_of(v[j]);
                    more += i + j < to && k > prefix;
                    equal += i + j < to && k == prefix;
                }
            }
            uint32_t all_more, all_equal;
            before_me(more, sums, all_more);
            before_me(equal, sums, all_equal);
            if (th == 0) { mine[0] = all_more; mine[1] = all_equal; }
            sync();
            for (int c = 0; c < rank; ++c) {
                at_more += remote(&mine[0], c);
                at_equal += remote(&mine[1], c);
            }
            sync();             // nobody leaves while its memory is read
        }
        for (int i0 = from; i0 < to; i0 += 4 * THREADS) {
            const int i = i0 + 4 * th;
            float v[4];
            load4(w, i, to, vectors, v);
            uint32_t k[4], mine_of = 0, all;            // how many above in the lower half, how many equal in the upper one
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                k[j] = key_of(v[j]);
                if (i + j < to) mine_of += (k[j] > prefix) | (k[j] == prefix) << 16;
            }
            const uint32_t front = before_me(mine_of, sums, all);
            uint32_t e = at_equal + (front >> 16), m = at_more + (front & 0xffff);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool above = i + j < to && k[j] > prefix, same = i + j < to && k[j] == prefix;
                if (above || (same && e < left)) {
                    const uint32_t place = min(m + min(e, left), static_cast<uint32_t>(need) - 1u);        // the least one but for weights that change meanwhile
                    kept[place] = i + j;
                    out[place] = v[j];
                }
                m += above;
                e += same;
            }
            at_more += all & 0xffff;
            at_equal += all >> 16;
        }
    }
    // the newest ones (all of them where nothing goes), and what is behind
    for (int i = need + rank * THREADS + th; i < a.keep; i += CTAS * THREADS) kept[i] = i < stay ? old + i - need : -1;
    for (int i = need + rank * THREADS + th; i < a.N; i += CTAS * THREADS) out[i] = i < stay ? w[old + i - need] : 0.f;
    if (h == 0 && rank == 0 && th == 0) a.lengths_out[b] = stay;
    if (__syncthreads_or(missing)) {            // all CTAs of a cluster see the same
        sync();
        if (rank == 0) select_around(a, own, other, b, n, w, kept, out, h == 0 ? a.lengths_out + b : nullptr, sums);
    }
}

// Eight lanes an entry: 16 bytes of keys or values each, then its steps.  STEP 0: into the other table's pages; 1: into the copy; 2: out of it.
template <int STEP>
__global__ void __launch_bounds__(256) kv4_move_kernel(const __grid_constant__ Evict a)
{
    constexpr int AHEAD = 4, WIDE = 32;       // entries that eight lanes have on their way; of a CTA side by side
    const int32_t* kept = dependent_begin(a.kept);
    const int lane = threadIdx.x & 7, h = blockIdx.y, D = a.l.D, half = D / 32, tiles = (a.keep + KV4_TILE - 1) / KV4_TILE;
    for (int b = blockIdx.z; b < a.from.B; b += gridDim.z) {
        const int stay = min(behind_wait<int32_t>(a.lengths_out)[b], a.keep);
        const long long head = static_cast<long long>(b) * a.l.H + h;
        unsigned char* copy = STEP == 0 ? nullptr : a.copy + head * tiles * a.l.tile;
        Kv4Table from = a.from, into = a.into;
        from.pages = behind_wait<int32_t>(a.from.pages);
        into.pages = behind_wait<int32_t>(a.into.pages);
        for (int r0 = blockIdx.x * WIDE * AHEAD + (threadIdx.x >> 3); r0 < stay; r0 += gridDim.x * WIDE * AHEAD) {
            unsigned char *src[AHEAD], *dst[AHEAD];
            int es[AHEAD], ed[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int r = r0 + k * WIDE, i = r < stay ? kept[head * a.keep + r] : -1;
                src[k] = dst[k] = nullptr;
                es[k] = i & (KV4_TILE - 1);
                ed[k] = r & (KV4_TILE - 1);
                if (i < 0 || (STEP > 0 && i == r)) continue;          // in place already
                const int ps = kv4_page_of(a.l, from, b, i), pd = kv4_page_of(a.l, into, b, r);
                if (ps < 0 || pd < 0) continue;
                unsigned char* held = STEP == 0 ? nullptr : copy + static_cast<long long>(r / KV4_TILE) * a.l.tile;
                src[k] = STEP == 2 ? held : kv4_tile_of(a.l, ps, h, i & (a.l.page - 1));
                dst[k] = STEP == 1 ? held : kv4_tile_of(a.l, pd, h, r & (a.l.page - 1));
                if (STEP == 2) es[k] = ed[k];
            }
            uint4 v[AHEAD];
            uint32_t s[AHEAD];
            // lanes below half: parts of the keys' row, the next ones of the values'
            auto part_of = [&](int e) {
                const int p = lane < half ? lane : lane - half;
                return lane < half ? kv4_key_row(e) * (D / 2) + 16 * p : KV4_TILE * (D / 2) + e * (D / 2) + 8 * kv4_value_part(D, e, 2 * p);
            };
            auto step_of = [&](int e) { return KV4_TILE * D + (lane < a.l.G ? e * a.l.G + lane : (KV4_TILE + e) * a.l.G + lane - a.l.G) * 4; };
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (src[k] && lane < 2 * half) v[k] = *reinterpret_cast<const uint4*>(src[k] + part_of(es[k]));
                if (src[k] && lane < 2 * a.l.G) s[k] = *reinterpret_cast<const uint32_t*>(src[k] + step_of(es[k]));
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (dst[k] && lane < 2 * half) *reinterpret_cast<uint4*>(dst[k] + part_of(ed[k])) = v[k];
                if (dst[k] && lane < 2 * a.l.G) *reinterpret_cast<uint32_t*>(dst[k] + step_of(ed[k])) = s[k];
            }
        }
    }
}

template <int CTAS>
int launch_select(const Evict& a, int B, cudaStream_t st) { return launch_clusters(kv4_select_kernel<CTAS>, CTAS, dim3(CTAS, a.l.H, B), dim3(THREADS), 0, st, a); }

}  // namespace
}  // namespace bs

using namespace bs;

extern "C" size_t bs_kv4_evict_workspace_bytes(const bs_kv4_cache* cache, int B, int keep, int into)
{
    Kv4 l;
    if (!cache || B <= 0 || keep <= 0 || keep > MOST_ROWS || !kv4_layout(*cache, l)) return 0;
    return into ? 0 : static_cast<size_t>(B) * l.H * ceil_div(keep, KV4_TILE) * l.tile;
}

extern "C" int bs_kv4_evict(const bs_kv4_cache* cache, const int32_t* table, long long table_pitch, int width, const int32_t* into, long long into_pitch, int into_width, int B,
                            const int32_t* lengths, const float* weights, long long weights_sequence, long long weights_head, int N, int keep, int recent, int32_t* lengths_out,
                            float* weights_out, int32_t* kept, void* workspace, size_t workspace_bytes, void* stream)
{
    Evict a{};
    if (!cache || !cache->data || !table || !lengths || !weights || !lengths_out || !weights_out || !kept || B <= 0 || width <= 0 || (table_pitch < width && (table_pitch != 0 || (!into && B > 1)))) return BS_ERR_INVALID_ARG;
    if (cache->type != BS_F16 && cache->type != BS_BF16) return BS_ERR_INVALID_ARG;
    if (cache->pages <= 0 || cache->heads <= 0 || cache->D <= 0 || cache->page <= 0 || cache->group <= 0) return BS_ERR_INVALID_ARG;
    if (N <= 0 || keep <= 0 || recent < 0 || recent > keep || weights_head < 0 || (weights_head > 0 && weights_head < N) || weights_sequence < 0) return BS_ERR_INVALID_ARG;
    if (into && (into_width <= 0 || into_pitch < into_width)) return BS_ERR_INVALID_ARG;
    if (!kv4_layout(*cache, a.l) || B > 65535 || N > MOST_ROWS || keep > MOST_ROWS) return BS_ERR_UNSUPPORTED;
    const long long most = static_cast<long long>(width) * a.l.page < N ? static_cast<long long>(width) * a.l.page : N, stays = keep < most ? keep : most;
    if (into && static_cast<long long>(into_width) * a.l.page < stays) return BS_ERR_INVALID_ARG;
    const size_t need = bs_kv4_evict_workspace_bytes(cache, B, keep, into != nullptr);
    if (need > 0 && (!workspace || workspace_bytes < need)) return BS_ERR_INVALID_ARG;
    if (!aligned16(cache->data) || !aligned16(workspace)) return BS_ERR_ALIGNMENT;
    a.from = {table, table_pitch, width, B};
    a.into = into ? Kv4Table{into, into_pitch, into_width, B} : a.from;
    a.lengths = lengths; a.weights = weights; a.w_sequence = weights_sequence; a.w_head = weights_head;
    a.N = N; a.keep = keep; a.recent = recent; a.inside = into == nullptr;
    a.lengths_out = lengths_out; a.weights_out = weights_out; a.kept = kept;
    a.copy = static_cast<unsigned char*>(workspace);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    // A CTA takes 16384 weights in about 10 us; more of them where there are so many and the heads leave SMs free.  By one, two and eight CTAs a head, with the moves:
    // 8 heads of 4096 entries 12.0, 19.5, 21.1 us; of 16384 23.0, 22.2, 25.5; of 32768 32.1, 30.9, 27.6; of 131072 103, 71, 46; 64 of 32768 83, 76, 82; 256 of 16384 99, 119, 224;
    // but 128 of 32768 120, 111, 157, and 32 of 131072 160, 129, 69, where the rule takes one and two.
    const long long heads = static_cast<long long>(a.l.H) * B, sms = device_sm_count();
    int rc = most <= 16384 || heads * 2 > sms ? launch_select<1>(a, B, st) : most <= 65536 || heads * 8 > sms ? launch_select<2>(a, B, st) : launch_select<MOST>(a, B, st);
    if (rc != BS_OK) return rc;
    const long long chunks = ceil_div_ll(stays, 128);
    const dim3 grid(static_cast<unsigned>(chunks < 4096 ? chunks : 4096), a.l.H, B);
    if (into) return launch_dependent(kv4_move_kernel<0>, grid, dim3(256), 0, st, a);
    rc = launch_dependent(kv4_move_kernel<1>, grid, dim3(256), 0, st, a);
    return rc == BS_OK ? launch_dependent(kv4_move_kernel<2>, grid, dim3(256), 0, st, a) : rc;
}
