// Attention of the newest tokens of each sequence over its entries in a cache of 4-bit keys and values: o = softmax(scale q K^T) V, one token or a few.
//
// Codes are exact in fp16 and are what the tensor cores multiply (mma.sync; eight rows of queries cost what one does): with c the codes, s and m a group's step
// and offset, a score is the sum over its groups of s (q . c) + m sum(q), scaled in 32 bits; the keys are never rounded.  An output is the sum over
// entries of (p s) c, p s in fp16 under a power of two of the row and the group, plus the sum of p m, in 32 bits.  A code costs a mask: as the last bits of an fp16
// number without an exponent it counts 2^-24, which the sums' scales take back.
//
// A warp takes 64 entries at a time, in one piece where the page allows, through two buffers of its own in shared memory, and keeps the running maximum, sum
// and outputs of eight or sixteen rows (query tokens times the heads that share keys) in registers.  Four warps of a CTA share a run of entries; the
// sequences are cut into runs of equal length for the whole grid, which every CTA finds by itself from the lengths; a second kernel joins runs, or, where they
// are short and few, clusters do.
//
// 64 sequences of up to 8192 entries, 32 heads over 8 of 128 channels: 66 us, 4.1 TB/s, where the bare stream takes 41 to 49 and the instructions (250 a tile of 16 entries
// and head, a third of them masks) 55 by themselves; 12 warps an SM issue in half of the cycles.  One sequence of 131072: 38 us, of 1000: 6.7.
#include "kv4.h"
#include "mma_kernel.cuh"
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int WARPS = 4, STAGES = 2, UNIT = 4;          // tiles of 16 entries that a warp takes at a time; with two 64 sequences take 20 % more
constexpr int LEAST = 8;                                // tiles of a run, at least
// CTAs of an SM, as registers and shared memory allow.  A fourth one needs 128 registers a thread and units of two tiles: 25 % more.
template <int D, int G> constexpr int ring_bytes() { return WARPS * STAGES * UNIT * KV4_TILE * (D + 8 * G); }
constexpr int ctas_of(int ring, int NT) { return (NT == 1 ? 3 : 2) < 227 * 1024 / (ring + 2048) ? (NT == 1 ? 3 : 2) : 227 * 1024 / (ring + 2048); }
constexpr int TEAMS = 8;                                // runs of a column, where a cluster joins them

struct Attend {
    Kv4 l;
    Kv4Table t;
    const int32_t* lengths;
    const int32_t* starts;      // null: one row of q a sequence
    const void* q;
    long long q_token, q_head;
    int T, Hq, per;             // rows of q, its heads, how many share a head of the cache
    FastDiv d_per, d_heads;
    float scale;                // times log2(e)
    void* out;                  // [T][Hq][D]
    float* part;                // [runs][R][D], and behind them
    float2* stat;               // [runs][R] maximum and sum
    int4* info;                 // [B] first run, runs of a column, columns, tiles of rows
    float* scores;              // [T][Hq][N], where weights are wanted
    float* lse;                 // [T][Hq]
    float* weights;
    long long w_sequence, w_head;
    int N;
    int slots;                  // CTAs that the GPU holds at a time
    int* status;
};

// Sequence b: entries, query tokens, tiles of entries and of rows.
struct Seq {
    int n, first, tq, tiles, rts;
    __device__ __forceinline__ Seq(const Attend& a, const int32_t* lengths, const int32_t* starts, int b, int R)
    {
        const long long room = min(static_cast<long long>(a.t.width) * a.l.page, 0x7fffff00LL);
        n = lengths[b];
        n = n < 0 ? 0 : n > room ? static_cast<int>(room) : n;
        first = b;
        tq = 1;
        if (starts) {
            first = min(max(starts[b], 0), a.T);
            tq = min(max(starts[b + 1], first), a.T) - first;
        }
        tiles = (n + KV4_TILE - 1) / KV4_TILE;
        rts = static_cast<int>((static_cast<long long>(tq) * a.per + R - 1) / R);
    }
};

__host__ __device__ __forceinline__ long long runs_of(long long columns, int slots) { return max((2 * columns + slots - 1) / slots, 1LL) * slots; }

__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// x 2^n, n from -252 to 254, by two factors, as 2^n alone may be out of range.  At least the smallest number and at most the largest one: an infinity times it stays
// one, and a zero a zero.
__device__ __forceinline__ float times_power(float x, int n)
{
    const int half = n >> 1;
    const float y = x * __uint_as_float(static_cast<uint32_t>(127 + half) << 23) * __uint_as_float(static_cast<uint32_t>(127 + n - half) << 23);
    return fminf(fmaxf(y, 0x1p-149f), 0x1.fffffep127f);
}
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ u64 f2_mul(u64 a, u64 b) { u64 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
// Nibbles i and i + 4 of x as pairs of fp16: bits at the end of a mantissa without an exponent are a number of 2^-24 each, four places up of 2^-20, exactly.
__device__ __forceinline__ void expand(uint32_t x, uint32_t (&v)[4])
{
    const uint32_t y = x >> 8;
    v[0] = x & 0x000f000fu;
    v[1] = x & 0x00f000f0u;
    v[2] = y & 0x000f000fu;
    v[3] = y & 0x00f000f0u;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Loads of what the bulk copies brought.  They may move, but not in front of the wait, whose statement their address comes out of, nor behind the next copy into
// the same place, in front of which the results of all of them are asked for.
template <int W> __device__ __forceinline__ void load_words(uint32_t at, uint32_t (&w)[W])
{
    if constexpr (W == 4) asm("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
    else if constexpr (W == 2) asm("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    else
#pragma unroll
        for (int i = 0; i < W; ++i) asm("ld.shared.u32 %0, [%1];" : "=r"(w[i]) : "r"(at + 4 * i));
}
// The D / 32 pieces of two bytes of a part of a values' row, two a word but for D = 96.
template <int C> constexpr int words_of = C == 3 ? 3 : C / 2;
template <int C> __device__ __forceinline__ void load_pieces(uint32_t at, uint32_t (&w)[words_of<C>])
{
    if constexpr (C == 3) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            uint16_t v;
            asm("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at + 2 * i));
            w[i] = v;
        }
    } else {
        load_words(at, w);
    }
}
template <int C> __device__ __forceinline__ uint32_t pair_of(const uint32_t (&a)[words_of<C>], const uint32_t (&b)[words_of<C>], int c)
{
    return C == 3 ? __byte_perm(a[c], b[c], 0x5410) : __byte_perm(a[c / 2], b[c / 2], c & 1 ? 0x7632 : 0x5410);
}

// TEAM: the runs of a column are the CTAs of a cluster, which joins them.
template <bool F16, int D, int G, int NT, bool TEAM>
__global__ void __launch_bounds__(WARPS * 32, ctas_of(ring_bytes<D, G>(), NT)) kv4_attend_kernel(const __grid_constant__ Attend a)
{
    typedef W4Type<F16> Ty;
    typedef W4Type<true> Half;
    // The weights' second fp16 term: without it outputs are off by up to 2^-12 of the weights' part of them, which an output of 11 bits would show and one of 8
    // does not (64 sequences: 73 us in place of 66, 131072 entries 41 in place of 38).
    constexpr bool TWO = F16;
    constexpr int R = 8 * NT, BLOCKS = D / 32, MT = D / 16, TILE = KV4_TILE * (D + 8 * G), PER_G = BLOCKS / G;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[WARPS][STAGES];
    __shared__ float2 stat[WARPS][R], whole[R];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tid = lane & 3;
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(&bars[warp][s], 1);
        fence_barrier_init();
        fence_proxy_async();
    }
    __syncwarp();
    dependent_begin(a.t.pages);
    const int32_t *lengths = behind_wait<int32_t>(a.lengths), *starts = a.starts ? behind_wait<int32_t>(a.starts) : nullptr, *table = behind_wait<int32_t>(a.t.pages);

    // the run that this CTA takes: its sequence, head, tile of rows and tiles of entries
    int b = 0, runs = 1, run = 0, column = 0, base = 0;
    {
        long long all = 0, columns = 0;
        for (int i = lane; i < a.t.B; i += 32) {
            const Seq s(a, lengths, starts, i, R);
            all += static_cast<long long>(s.tiles) * s.rts * a.l.H;
            columns += s.rts * a.l.H;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            all += __shfl_xor_sync(0xffffffffu, all, d);
            columns += __shfl_xor_sync(0xffffffffu, columns, d);
        }
        // as many runs as fill the GPU once, or as often as it takes for half of them to be cuts: every column may end in a short one
        const long long target = max(runs_of(columns, a.slots) - columns, 1LL);
        const int chunk = static_cast<int>(min(max((all + target - 1) / target, static_cast<long long>(LEAST)), 1LL << 30));
        int before = 0;
        bool found = false;
        for (int i0 = 0; i0 < a.t.B && !found; i0 += 32) {
            int n = 0, r = 1, c = 1;
            if (i0 + lane < a.t.B) {
                const Seq s(a, lengths, starts, i0 + lane, R);
                r = TEAM ? TEAMS : max(1, (s.tiles + chunk - 1) / chunk);
                c = s.rts * a.l.H;
                n = r * c;
            }
            int sum = n;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int v = __shfl_up_sync(0xffffffffu, sum, d);
                if (lane >= d) sum += v;
            }
            const int from = before + sum - n;
            const unsigned here = __ballot_sync(0xffffffffu, static_cast<int>(blockIdx.x) >= from && static_cast<int>(blockIdx.x) < from + n);
            if (here) {
                const int who = __ffs(here) - 1;
                b = i0 + who;
                runs = __shfl_sync(0xffffffffu, r, who);
                base = __shfl_sync(0xffffffffu, from, who);
                c = __shfl_sync(0xffffffffu, c, who);
                run = TEAM ? (blockIdx.x - base) % TEAMS : (blockIdx.x - base) / c;
                column = TEAM ? (blockIdx.x - base) / TEAMS : (blockIdx.x - base) - run * c;
                found = true;
            }
            before += __shfl_sync(0xffffffffu, sum, 31);
        }
        if (!found) return;
    }
    const Seq s(a, lengths, starts, b, R);
    auto token_of = [&](int r) { return fdiv(r, a.d_per); };                // of the sequence's query tokens, the one of row r
    const int h = column - fdiv(column, a.d_heads) * a.l.H, r0 = fdiv(column, a.d_heads) * R, rows = s.tq * a.per;
    auto row_of = [&](int r) { return static_cast<long long>(s.first + token_of(r)) * a.Hq + h * a.per + r - token_of(r) * a.per; };       // of q and out
    if (!TEAM && a.info && column == 0 && run == 0 && threadIdx.x == 0) a.info[b] = make_int4(base, runs, s.rts * a.l.H, 0);

    // how many entries a row sees; rows behind the last one see all and are dropped
    int limit[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = r0 + n * 8 + 2 * tid + i;
            limit[n][i] = r < rows ? s.n - s.tq + token_of(r) + 1 : s.n;
        }
    const int least = s.n - s.tq + token_of(r0) + 1;                              // entries that all rows see
    const int most = s.n - s.tq + token_of(min(rows - 1, r0 + R - 1)) + 1;        // and that any row sees
    const int tiles = max(0, (min(most, s.n) + KV4_TILE - 1) / KV4_TILE);
    const int t0 = min(tiles, static_cast<int>(static_cast<long long>(s.tiles) * run / runs)), t1 = min(tiles, static_cast<int>(static_cast<long long>(s.tiles) * (run + 1) / runs));
    const int unit = min(UNIT, max(1, (t1 - t0 + WARPS - 1) / WARPS));
    const int units = (t1 - t0 + unit - 1) / unit, mine = units > warp ? (units - warp + WARPS - 1) / WARPS : 0;

    // copies ahead: lane 4 i + j looks up the page of tile j of the warp's unit i, eight units at a time
    unsigned char* ring = smem + warp * STAGES * UNIT * TILE;
    const uint32_t ring_at = smem_u32(ring);
    const int log_tiles = a.l.log_page - 4, in_page = (1 << log_tiles) - 1;        // of a page
    const int32_t* row = table + b * a.t.pitch;
    const unsigned char* mine_at = a.l.data + h * a.l.head;
    int page = -1;
    unsigned there = 0, flags = 0;          // which of the eight units' tiles have a page; the same of the stages, four bits each
    auto issue = [&](int k) {
        if ((k & 7) == 0) {
            const int t = t0 + (warp + WARPS * (k + (lane >> 2))) * unit + (lane & 3);
            page = -1;
            if ((lane & 3) < unit && t < t1) page = row[t >> log_tiles];
            if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.l.pages)) page = -1;
            there = __ballot_sync(0xffffffffu, page >= 0);
        }
        const int stage = k % STAGES, f = t0 + (warp + WARPS * k) * unit, count = min(unit, t1 - f);
        flags = (flags & ~(15u << 4 * stage)) | (there >> 4 * (k & 7) & 15u) << 4 * stage;
        if (lane == 0) mbar_expect_tx(&bars[warp][stage], count * TILE);
        __syncwarp();
        const int j = lane & 3, t = f + j;
        if ((lane >> 2) == (k & 7) && j < count && (j == 0 || (t & in_page) == 0)) {
            const int len = min(count - j, in_page + 1 - (t & in_page));
            const unsigned char* from = mine_at + max(page, 0) * a.l.whole + (t & in_page) * TILE;
            mm_bulk(ring + (stage * UNIT + j) * TILE, from, len * TILE, &bars[warp][stage]);
        }
    };
#pragma unroll
    for (int k = 0; k < STAGES; ++k)
        if (k < mine) issue(k);

    // queries as fragments: row gid of each tile, the channels in the order of the keys' words.  A power of two brings a row's largest value to 2^13 and more, so that its
    // others fit fp16 exactly, those that meet codes of sixteenfold weight divided by sixteen, but for values below 2^-23 (bf16: 2^-26) of the largest, which
    // may lose 2^-34 of it
    uint32_t qf[NT][BLOCKS * 2][2];
    float factor[NT][2], qsum[G][NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = r0 + n * 8 + gid;
        uint4 raw[BLOCKS];
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) raw[k] = make_uint4(0, 0, 0, 0);
        if (r < rows) {
            const int i = token_of(r);
            const uint16_t* q = behind_wait<uint16_t>(a.q) + (s.first + i) * a.q_token + (h * a.per + r - i * a.per) * a.q_head + 8 * tid;
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k) raw[k] = *reinterpret_cast<const uint4*>(q + 32 * k);
        }
        uint32_t big = 0;
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w = word_of(raw[k], j);
                big = max(big, max(__float_as_uint(fabsf(Ty::lo(w))), __float_as_uint(fabsf(Ty::hi(w)))));
            }
        big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
        const int e = min(max(static_cast<int>(big >> 23) - 127, -112), 126), down = e - 13;       // the largest value's exponent becomes 13
        const float up = __uint_as_float(static_cast<uint32_t>(127 - down) << 23);
        float sums[G];
#pragma unroll
        for (int g = 0; g < G; ++g) sums[g] = 0.f;
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[2 * j] = Ty::lo(word_of(raw[k], j)) * up;
                x[2 * j + 1] = Ty::hi(word_of(raw[k], j)) * up;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[k / PER_G] += x[j];
            // the odd pairs meet codes that count sixteen times as much
            qf[n][2 * k][0] = half2_of(x[0], x[4]);
            qf[n][2 * k][1] = half2_of(x[1] * 0.0625f, x[5] * 0.0625f);
            qf[n][2 * k + 1][0] = half2_of(x[2], x[6]);
            qf[n][2 * k + 1][1] = half2_of(x[3] * 0.0625f, x[7] * 0.0625f);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            sums[g] += __shfl_xor_sync(0xffffffffu, sums[g], 1);
            sums[g] += __shfl_xor_sync(0xffffffffu, sums[g], 2);
        }
        // from the rows' lanes to the columns'
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int from = 4 * (2 * tid + i);
            factor[n][i] = times_power(a.scale, __shfl_sync(0xffffffffu, down, from) + 24);        // sums are in units of 2^-24
#pragma unroll
            for (int g = 0; g < G; ++g) qsum[g][n][i] = __shfl_sync(0xffffffffu, sums[g], from) * 0x1p-24f;
        }
    }

    // Products p s of a row and group of channels are scaled by a power of two that keeps them below 2^15 and the largest one that was met above 1, so that fp16 loses no
    // more than 2^-25 of that one, whatever steps the entries without weight and the other groups have.  cap: the bits of what stands for 2^15; the outputs' units follow.
    constexpr int LEAST_CAP = 24 << 23;         // 2^-103
    float o[MT][NT][4], offs[G][NT][2], top[NT][2], total[NT][2];
    int cap[G][NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            top[n][i] = -INFINITY;
            total[n][i] = 0.f;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                offs[g][n][i] = 0.f;
                cap[g][n][i] = LEAST_CAP;
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) o[m][n][i] = o[m][n][2 + i] = 0.f;
        }
    const int place[2] = {(gid >> 1) + 4 * (gid & 1), (gid >> 1) + 4 * (gid & 1) + 8};     // entries of rows gid and gid + 8 of a fragment
    // where a lane reads in a tile: its rows of the keys, their steps, and its part of the values' rows tid, tid + 4, tid + 8, tid + 12 (whose parts lie alike)
    uint32_t key_at[2], step_at[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        key_at[i] = kv4_key_row(place[i]) * (D / 2) + tid * (D / 8);
        step_at[i] = place[i] * (4 * G);
    }
    const uint32_t value_at = tid * (D / 2) + kv4_value_part(D, tid, gid) * (D / 16);

    auto unit_of = [](int cap) { return __uint_as_float((269u << 23) - static_cast<uint32_t>(cap)); };          // 2^15 / cap

    // A whole unit that all rows see, in halves where registers would not do (64 sequences, 4 tokens, fp16, groups of 64: 180 us whole, 170 in halves), or one tile `at`
    // of any: code that runs once or twice should be short, it comes from memory.
    constexpr int AT_ONCE = G * NT < 4 ? UNIT : UNIT / 2;
    auto take = [&](int k, int at, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        constexpr int TILES = MASKED ? 1 : AT_ONCE;
        const int stage = k % STAGES, first = (t0 + (warp + WARPS * k) * unit + at) * KV4_TILE;
        const bool there_is = flags >> (4 * stage + at) & 1;
        uint32_t unit_at = ring_at + (stage * UNIT + at) * TILE;
        asm volatile("" : "+r"(unit_at) : : "memory");
        float p[TILES][NT][4], high[NT][2], step_top[G];
        uint32_t value_step[TILES][2][G];
#pragma unroll
        for (int n = 0; n < NT; ++n) high[n][0] = high[n][1] = -INFINITY;
#pragma unroll
        for (int g = 0; g < G; ++g) step_top[g] = 0.f;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const uint32_t tile = unit_at + t * TILE;
            uint32_t key[2][BLOCKS], step[2][G];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                load_words(tile + key_at[i], key[i]);
                load_words(tile + KV4_TILE * D + step_at[i], step[i]);
            }
            float sum[NT][4];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float acc[NT][4], more[NT][4];         // two sums, so that half as many products wait for one another
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][i] = more[n][i] = 0.f;
#pragma unroll
                for (int k2 = g * PER_G; k2 < (g + 1) * PER_G; ++k2) {
                    uint32_t x[4], y[4];
                    expand(key[0][k2], x);
                    expand(key[1][k2], y);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        Half::mma(acc[n], x[0], y[0], x[1], y[1], qf[n][2 * k2][0], qf[n][2 * k2][1]);
                        Half::mma(more[n], x[2], y[2], x[3], y[3], qf[n][2 * k2 + 1][0], qf[n][2 * k2 + 1][1]);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][i] += more[n][i];
                const float s0 = Ty::lo(step[0][g]), s1 = Ty::lo(step[1][g]), m0 = Ty::hi(step[0][g]), m1 = Ty::hi(step[1][g]);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float c0 = m0 * qsum[g][n][i], c1 = m1 * qsum[g][n][i];
                        sum[n][i] = g == 0 ? fmaf(acc[n][i], s0, c0) : sum[n][i] + fmaf(acc[n][i], s0, c0);
                        sum[n][2 + i] = g == 0 ? fmaf(acc[n][2 + i], s1, c1) : sum[n][2 + i] + fmaf(acc[n][2 + i], s1, c1);
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = sum[n][i];
                    if (MASKED && (first + t * KV4_TILE + place[i >> 1] >= limit[n][i & 1] || !there_is)) v = -INFINITY;
                    p[t][n][i] = v;
                    high[n][i & 1] = fmaxf(high[n][i & 1], v);
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                load_words(tile + KV4_TILE * D + 64 * G + step_at[i], value_step[t][i]);
                if (MASKED && (first + t * KV4_TILE + place[i] >= s.n || !there_is))
#pragma unroll
                    for (int g = 0; g < G; ++g) value_step[t][i][g] = 0;
#pragma unroll
                for (int g = 0; g < G; ++g) step_top[g] = fmaxf(step_top[g], Ty::lo(value_step[t][i][g]));
            }
        }
        if (a.scores) {
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = r0 + n * 8 + 2 * tid + (i & 1), e = first + t * KV4_TILE + place[i >> 1];
                        if (r < rows && e < a.N)
                            a.scores[row_of(r) * a.N + e] = p[t][n][i] * factor[n][i & 1];
                    }
        }
        // Weights are relative to a maximum, a whole number, that is replaced only when a score is above it by 8 (weights then stay below 2^8); what is there so far
        // shrinks by a power of two, which the outputs' units take.  The units are looked at where the lane's largest weight times its largest step asks for it.
        bool grown = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float over = fmaf(high[n][i], factor[n][i], -top[n][i]), most = exp2_of(over);
                grown |= over > 8.f;
#pragma unroll
                for (int g = 0; g < G; ++g) grown |= most * step_top[g] > __int_as_float(cap[g][n][i]);
            }
        if (__any_sync(0xffffffffu, grown)) {
            // the lane's largest weight times its least step is below what its entries have: often enough to find the units by; else they are looked at one by one
            float step_least[G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                step_least[g] = step_top[g];
#pragma unroll
                for (int t = 0; t < TILES; ++t) step_least[g] = fminf(step_least[g], fminf(Ty::lo(value_step[t][0][g]), Ty::lo(value_step[t][1][g])));
            }
            auto of_all = [](float v) {           // the largest of the lanes that have the same rows
#pragma unroll
                for (int d = 4; d < 32; d *= 2) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
                return v;
            };
            auto peak_of = [&](int g, int n, int i) {
                float v = 0.f;
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int j = 0; j < 2; ++j) v = fmaxf(v, exp2_of(fmaf(p[t][n][2 * j + i], factor[n][i], -top[n][i])) * Ty::lo(value_step[t][j][g]));
                return v;
            };
            auto exponent_of = [](float v) { return min(static_cast<int>(__float_as_uint(v) >> 23), 239); };
            auto outputs_by = [&](int g, int n, int i, int exponent) {
                const float f = __uint_as_float(static_cast<uint32_t>(max(127 + exponent, 0)) << 23);
#pragma unroll
                for (int m = 2 * g * PER_G; m < 2 * (g + 1) * PER_G; ++m) {
                    o[m][n][i] *= f;
                    o[m][n][2 + i] *= f;
                }
            };
            bool tight = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float v = of_all(high[n][i] * factor[n][i]);
                    v = v > top[n][i] + 8.f ? floorf(v) : top[n][i];
                    const int fall = static_cast<int>(fmaxf(top[n][i] - v, -255.f));          // -255 where there was no maximum, too
                    const float f = __uint_as_float(static_cast<uint32_t>(max(127 + fall, 0)) << 23), most = exp2_of(v == -INFINITY ? v : fmaf(high[n][i], factor[n][i], -v));
                    top[n][i] = v;
                    total[n][i] *= f;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        offs[g][n][i] *= f;
                        const float least = MASKED ? peak_of(g, n, i) : most * step_least[g];
                        const int had = (cap[g][n][i] >> 23) + fall, has = max(max(had, LEAST_CAP >> 23), exponent_of(of_all(least)) + 15);
                        cap[g][n][i] = has << 23;
                        tight |= !MASKED && most * step_top[g] > __int_as_float(cap[g][n][i]);
                        if (k + at > 0) outputs_by(g, n, i, had - has);
                    }
                }
            if (!MASKED && __any_sync(0xffffffffu, tight)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int g = 0; g < G; ++g) {
                            const int had = cap[g][n][i] >> 23, e = exponent_of(of_all(peak_of(g, n, i))), has = e >= had ? e + 15 : had;
                            cap[g][n][i] = has << 23;
                            outputs_by(g, n, i, had - has);
                        }
            }
        }
        float from[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) from[n][i] = top[n][i] == -INFINITY ? 0.f : -top[n][i];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const uint32_t tile = unit_at + t * TILE;
            uint32_t word[4][words_of<BLOCKS>];
#pragma unroll
            for (int i = 0; i < 4; ++i) load_pieces<BLOCKS>(tile + KV4_TILE * (D / 2) + value_at + i * 2 * D, word[i]);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[t][n][i] = exp2_of(fmaf(p[t][n][i], factor[n][i & 1], from[n][i & 1]));
                    total[n][i & 1] += p[t][n][i];
                }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float st = Ty::lo(value_step[t][i][g]), off = Ty::hi(value_step[t][i][g]);
                    const int e = first + t * KV4_TILE + place[i];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const float p0 = p[t][n][2 * i], p1 = p[t][n][2 * i + 1];
                        uint32_t w0, w1;
                        f2_split(f2_mul(f2_mul(f2_pack(__float_as_uint(p0), __float_as_uint(p1)), f2_pack(__float_as_uint(st), __float_as_uint(st))),
                                        f2_pack(__float_as_uint(unit_of(cap[g][n][0])), __float_as_uint(unit_of(cap[g][n][1])))), w0, w1);
                        offs[g][n][0] = MASKED && e >= limit[n][0] ? offs[g][n][0] : fmaf(p0, off, offs[g][n][0]);
                        offs[g][n][1] = MASKED && e >= limit[n][1] ? offs[g][n][1] : fmaf(p1, off, offs[g][n][1]);
                        const uint32_t w = half2_of(__uint_as_float(w0), __uint_as_float(w1));
                        hi[n][i] = transposed(w);
                        if (TWO) lo[n][i] = transposed(half2_of(__uint_as_float(w0) - Half::lo(w), __uint_as_float(w1) - Half::hi(w)));
                    }
                }
#pragma unroll
                for (int c = g * PER_G; c < (g + 1) * PER_G; ++c) {
                    uint32_t x[4], y[4];
                    expand(pair_of<BLOCKS>(word[0], word[1], c), x);
                    expand(pair_of<BLOCKS>(word[2], word[3], c), y);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        Half::mma(o[2 * c][n], x[0], x[1], y[0], y[1], hi[n][0], hi[n][1]);
                        Half::mma(o[2 * c + 1][n], x[2], x[3], y[2], y[3], hi[n][0], hi[n][1]);
                        if (TWO) {
                            Half::mma(o[2 * c][n], x[0], x[1], y[0], y[1], lo[n][0], lo[n][1]);
                            Half::mma(o[2 * c + 1][n], x[2], x[3], y[2], y[3], lo[n][0], lo[n][1]);
                        }
                    }
                }
            }
        }
    };
    for (int k = 0; k < mine; ++k) {
        const int stage = k % STAGES;
        if (__any_sync(0xffffffffu, !mm_wait(&bars[warp][stage], k / STAGES & 1))) {
            // a wait that ran out: no more copies, and those on their way get as long again, since the outputs go where they land
            if (lane == 0) atomicOr(a.status, STATUS_TIMEOUT);
            for (int i = k; i < mine && i < k + STAGES; ++i) mm_wait(&bars[warp][i % STAGES], i / STAGES & 1);
            __syncwarp();
            break;
        }
        const int f = t0 + (warp + WARPS * k) * unit, count = min(unit, t1 - f);
        const unsigned whole = (1u << count) - 1u;
        if (count == UNIT && (f + count) * KV4_TILE <= least && (flags >> 4 * stage & whole) == whole)
#pragma unroll 1
            for (int i = 0; i < UNIT; i += AT_ONCE) take(k, i, std::false_type());
        else
#pragma unroll 1
            for (int i = 0; i < count; ++i) take(k, i, std::true_type());
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) asm volatile("" : "+f"(o[m][n][0]), "+f"(o[m][n][1]), "+f"(o[m][n][2]), "+f"(o[m][n][3]) : : "memory");
        __syncwarp();
        if (k + STAGES < mine) issue(k + STAGES);
    }

    // the warps' parts: rows of outputs [R][D], put together in the ring's memory
    __syncthreads();
    constexpr int PITCH = D + 4;
    float *outs = reinterpret_cast<float*>(smem), *joined = outs + WARPS * R * PITCH;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int d = 4; d < 32; d *= 2) {
                total[n][i] += __shfl_xor_sync(0xffffffffu, total[n][i], d);
#pragma unroll
                for (int g = 0; g < G; ++g) offs[g][n][i] += __shfl_xor_sync(0xffffffffu, offs[g][n][i], d);
            }
            const int r = n * 8 + 2 * tid + i;
            if (gid == 0) stat[warp][r] = make_float2(top[n][i], total[n][i]);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float back = __int_as_float(cap[m / (2 * PER_G)][n][i] - (15 << 23));          // and codes were in units of 2^-24, in rows gid + 8 of 2^-20
                outs[(warp * R + r) * PITCH + 16 * m + gid] = fmaf(o[m][n][i] * 0x1p24f, back, offs[m / (2 * PER_G)][n][i]);
                outs[(warp * R + r) * PITCH + 16 * m + gid + 8] = fmaf(o[m][n][2 + i] * 0x1p20f, back, offs[m / (2 * PER_G)][n][i]);
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < R * (D / 4); i += WARPS * 32) {
        const int r = i / (D / 4), d = i % (D / 4) * 4, row = r0 + r;
        float m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) m = fmaxf(m, stat[w][r].x);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = stat[w][r].x == -INFINITY ? 0.f : exp2_of(stat[w][r].x - m);
            const float4 x = *reinterpret_cast<const float4*>(outs + (w * R + r) * PITCH + d);
            if (stat[w][r].x == -INFINITY && stat[w][r].y == 0.f) continue;        // saw nothing
            sum = fmaf(stat[w][r].y, f, sum);
            v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
        }
        if (TEAM) {
            *reinterpret_cast<float4*>(joined + r * D + d) = v;
            if (d == 0) whole[r] = make_float2(m, sum);
            continue;
        }
        if (row >= rows) continue;
        if (runs == 1) {
            const long long at = row_of(row);
            const float inverse = sum == 0.f ? 0.f : 1.f / sum;
            uint32_t* to = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + at * D + d);
            *reinterpret_cast<uint2*>(to) = make_uint2(Ty::round2(v.x * inverse, v.y * inverse), Ty::round2(v.z * inverse, v.w * inverse));
            if (a.scores && d == 0) a.lse[at] = sum == 0.f ? INFINITY : m + log2f(sum);
        } else {
            *reinterpret_cast<float4*>(a.part + (static_cast<long long>(blockIdx.x) * R + r) * D + d) = v;
            if (d == 0) a.stat[static_cast<long long>(blockIdx.x) * R + r] = make_float2(m, sum);
        }
    }
    if (TEAM) {
        __syncwarp();
        mm_cluster_sync();
        for (int i = run * (WARPS * 32) + threadIdx.x; i < R * (D / 4); i += TEAMS * WARPS * 32) {
            const int r = i / (D / 4), d = i % (D / 4) * 4, row = r0 + r;
            float2 st[TEAMS];
            float4 x[TEAMS], v = make_float4(0.f, 0.f, 0.f, 0.f);
            float m = -INFINITY, sum = 0.f;
#pragma unroll
            for (int c = 0; c < TEAMS; ++c) {
                uint32_t at;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&whole[r])), "r"(c));
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(st[c].x), "=f"(st[c].y) : "r"(at));
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(joined + r * D + d)), "r"(c));
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[c].x), "=f"(x[c].y), "=f"(x[c].z), "=f"(x[c].w) : "r"(at));
            }
#pragma unroll
            for (int c = 0; c < TEAMS; ++c) m = fmaxf(m, st[c].x);
#pragma unroll
            for (int c = 0; c < TEAMS; ++c) {
                const bool empty = st[c].x == -INFINITY && st[c].y == 0.f;
                const float f = empty ? 0.f : exp2_of(st[c].x - m);
                sum = fmaf(st[c].y, f, sum);
                v.x = fmaf(x[c].x, f, v.x); v.y = fmaf(x[c].y, f, v.y); v.z = fmaf(x[c].z, f, v.z); v.w = fmaf(x[c].w, f, v.w);
            }
            if (row >= rows) continue;
            const long long at = row_of(row);
            const float inverse = sum == 0.f ? 0.f : 1.f / sum;
            uint32_t* to = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + at * D + d);
            *reinterpret_cast<uint2*>(to) = make_uint2(Ty::round2(v.x * inverse, v.y * inverse), Ty::round2(v.z * inverse, v.w * inverse));
            if (a.scores && d == 0) a.lse[at] = sum == 0.f ? INFINITY : m + log2f(sum);
        }
        __syncwarp();
        mm_cluster_sync();          // nobody leaves while its memory is read
    }
}

// Joins the runs of each row that was cut: a CTA a row of q and head, its warps the runs in turn: eight where columns are cut into sixteen and more (131072 entries 38.0 us,
// with four 39.9), four else (64 sequences of 8192 105.0, with eight 107.7; 128 of 2048 76.8 and 82.8; 4 of 32768, about where the two meet, 36.6 and 36.2).
constexpr int JOINERS = 8;
template <bool F16, int D>
__global__ void __launch_bounds__(JOINERS * 32) kv4_join_kernel(const __grid_constant__ Attend a, int R, int all)
{
    typedef W4Type<F16> Ty;
    __shared__ float4 outs[JOINERS][D / 4];
    __shared__ float total[JOINERS];
    dependent_begin(a.out);
    const int32_t* starts = a.starts ? behind_wait<int32_t>(a.starts) : nullptr;
    const int t = blockIdx.x, b = kv4_sequence_of(starts, a.t.B, t), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, joiners = blockDim.x >> 5;
    if (starts && (t < starts[b] || t >= starts[b + 1])) return;
    const int i = starts ? t - max(starts[b], 0) : 0;
    const int4 info = *behind_wait<int4>(a.info + b);
    if (info.y <= 1) return;            // whole already
    const int hq = blockIdx.y, h = hq / a.per, row = i * a.per + hq % a.per, r = row % R;
    const long long first = info.x + static_cast<long long>(row / R) * a.l.H + h;
    // starts in disorder may leave a sequence without its runs
    if (info.x < 0 || info.z <= 0 || first + (info.y - 1LL) * info.z >= all) return;
    const float2* stats = behind_wait<float2>(a.stat);
    const float* part = behind_wait<float>(a.part);
    float m = -INFINITY;
    for (int k = lane; k < info.y; k += 32) m = fmaxf(m, stats[(first + static_cast<long long>(k) * info.z) * R + r].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    const bool live = lane < D / 4;
#pragma unroll 4
    for (int k = warp; k < info.y; k += joiners) {
        const long long at = (first + static_cast<long long>(k) * info.z) * R + r;
        const float2 st = stats[at];
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (live) x = *reinterpret_cast<const float4*>(part + at * D + 4 * lane);
        const bool empty = st.x == -INFINITY && st.y == 0.f;
        const float f = empty ? 0.f : exp2_of(st.x - m);
        sum = fmaf(st.y, f, sum);
        v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
    }
    if (live) outs[warp][lane] = v;
    if (lane == 0) total[warp] = sum;
    __syncthreads();
    if (warp > 0) return;
    sum = total[0];
#pragma unroll
    for (int w = 1; w < joiners; ++w) sum += total[w];
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
    const long long at = static_cast<long long>(t) * a.Hq + hq;
    if (live) {
        v = outs[0][lane];
#pragma unroll
        for (int w = 1; w < joiners; ++w) { v.x += outs[w][lane].x; v.y += outs[w][lane].y; v.z += outs[w][lane].z; v.w += outs[w][lane].w; }
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at * D + 4 * lane) =
            make_uint2(Ty::round2(v.x * inverse, v.y * inverse), Ty::round2(v.z * inverse, v.w * inverse));
    }
    if (a.scores && lane == 0) a.lse[at] = sum == 0.f ? INFINITY : m + log2f(sum);
}

// What each entry got: the sum over the rows that share its head of exp2(score - lse).  Four threads an entry take every fourth row, their sums are added in order:
// the same bits every time.
__global__ void __launch_bounds__(256) kv4_weights_kernel(const __grid_constant__ Attend a)
{
    __shared__ float parts[4][64];
    dependent_begin(a.weights);
    const int32_t *lengths = behind_wait<int32_t>(a.lengths), *starts = a.starts ? behind_wait<int32_t>(a.starts) : nullptr;
    const int h = blockIdx.y, group = threadIdx.x >> 6, mine = threadIdx.x & 63;
    const float *lse = behind_wait<float>(a.lse), *scores = behind_wait<float>(a.scores);
    for (int b = blockIdx.z; b < a.t.B; b += gridDim.z) {
        const Seq s(a, lengths, starts, b, 8);
        const int n = min(s.n, a.N), rows = s.tq * a.per;
        for (int e0 = blockIdx.x * 64; e0 < n; e0 += gridDim.x * 64) {
            const int e = e0 + mine;
            float w = 0.f;
            if (e < n) {
                const int first = max(0, e - (s.n - s.tq)) * a.per;         // rows before it do not see the entry
#pragma unroll 4
                for (int r = first + group; r < rows; r += 4) {
                    const int i = fdiv(r, a.d_per);
                    const long long row = static_cast<long long>(s.first + i) * a.Hq + h * a.per + r - i * a.per;
                    w += exp2_of(scores[row * a.N + e] - lse[row]);
                }
            }
            parts[group][mine] = w;
            __syncthreads();
            if (group == 0 && e < n) a.weights[b * a.w_sequence + h * a.w_head + e] += (parts[0][mine] + parts[1][mine]) + (parts[2][mine] + parts[3][mine]);
            __syncthreads();
        }
    }
}

// Tiles of rows and runs that a call may have, and its workspace.  With weights the scores of all rows, 4 T Hq N bytes, are the most of it.
struct Plan {
    int NT, slots;
    bool team, join;            // joined by clusters; or, where a sequence may be longer than a run, by a second launch
    long long runs, cuts;       // and of a column, about
    size_t part, stat, info, lse, scores;
    size_t bytes() const { return part + stat + info + lse + scores; }
};
bool plan(const Kv4& l, int B, int T, int Hq, bool starts, int width, int N, int sms, Plan& p)
{
    const int per = Hq / l.H;
    const long long rows = starts ? ceil_div_ll(T, B) * per : per;
    p.NT = rows > 8 ? 2 : 1;
    const int R = 8 * p.NT;
    p.slots = sms * ctas_of(WARPS * STAGES * UNIT * l.tile, p.NT);
    const long long columns = starts ? l.H * (ceil_div_ll(static_cast<long long>(T) * per, R) + B) : static_cast<long long>(l.H) * B * ceil_div(per, R);
    const long long cuts = ceil_div_ll(static_cast<long long>(width) * l.page, LEAST * KV4_TILE), most = runs_of(columns, p.slots);
    p.runs = cuts < most / columns + 1 ? (columns * cuts < most ? columns * cuts : most) : most;
    // By the width of the table, as lengths are on the device and change under a captured call.  Few columns, of sequences so short that runs for the whole GPU would spare a warp no more than two turns of 1.2 us: a cluster a column, which spares the second
    // launch (1 x 1000 entries 8.8 us with it, 6.7 without)
    const long long tiles = ceil_div_ll(static_cast<long long>(width) * l.page, KV4_TILE), turn = WARPS * UNIT;
    p.team = columns * TEAMS <= p.slots && ceil_div_ll(tiles, TEAMS * turn) <= ceil_div_ll(tiles * columns, p.slots * turn) + 2;
    if (p.team) p.runs = columns * TEAMS;
    if (p.runs > 0x7fffffff / (R * 2)) return false;
    auto up = [](long long bytes) { return static_cast<size_t>((bytes + 255) / 256 * 256); };
    p.join = !p.team && cuts > 1;
    p.cuts = p.runs / columns;
    p.part = p.join ? up(p.runs * R * l.D * 4) : 0;
    p.stat = p.join ? up(p.runs * R * 8) : 0;
    p.info = p.join ? up(static_cast<long long>(B) * 16) : 0;
    p.lse = N > 0 ? up(static_cast<long long>(T) * Hq * 4) : 0;
    p.scores = N > 0 ? up(static_cast<long long>(T) * Hq * N * 4) : 0;
    return true;
}

template <bool F16, int D, int G, int NT>
int launch(const Attend& a, const Plan& p, cudaStream_t st)
{
    constexpr int ring = ring_bytes<D, G>(), parts = (WARPS * (D + 4) + D) * 8 * NT * 4, smem = ring > parts ? ring : parts;
    const dim3 grid(static_cast<unsigned>(p.runs)), block(WARPS * 32);
    if (p.team)
        return allow_shared<kv4_attend_kernel<F16, D, G, NT, true>>(smem) ? launch_clusters(kv4_attend_kernel<F16, D, G, NT, true>, TEAMS, grid, block, smem, st, a) : BS_ERR_CUDA;
    return allow_shared<kv4_attend_kernel<F16, D, G, NT, false>>(smem) ? launch_dependent(kv4_attend_kernel<F16, D, G, NT, false>, grid, block, smem, st, a) : BS_ERR_CUDA;
}
template <bool F16, int D, int G>
int launch_rows(const Attend& a, const Plan& p, cudaStream_t st) { return p.NT == 1 ? launch<F16, D, G, 1>(a, p, st) : launch<F16, D, G, 2>(a, p, st); }
template <bool F16>
int launch_form(const Attend& a, const Plan& p, cudaStream_t st)
{
    int rc;
    if (a.l.D == 64) rc = a.l.G == 1 ? launch_rows<F16, 64, 1>(a, p, st) : launch_rows<F16, 64, 2>(a, p, st);
    else if (a.l.D == 96) rc = a.l.G == 1 ? launch_rows<F16, 96, 1>(a, p, st) : launch_rows<F16, 96, 3>(a, p, st);
    else rc = a.l.G == 1 ? launch_rows<F16, 128, 1>(a, p, st) : a.l.G == 2 ? launch_rows<F16, 128, 2>(a, p, st) : launch_rows<F16, 128, 4>(a, p, st);
    if (rc != BS_OK) return rc;
    if (p.join) {
        const dim3 grid(a.T, a.Hq), block(p.cuts >= 16 ? JOINERS * 32 : JOINERS * 16);
        rc = a.l.D == 64 ? launch_dependent(kv4_join_kernel<F16, 64>, grid, block, 0, st, a, 8 * p.NT, static_cast<int>(p.runs))
             : a.l.D == 96 ? launch_dependent(kv4_join_kernel<F16, 96>, grid, block, 0, st, a, 8 * p.NT, static_cast<int>(p.runs))
                           : launch_dependent(kv4_join_kernel<F16, 128>, grid, block, 0, st, a, 8 * p.NT, static_cast<int>(p.runs));
    }
    if (rc == BS_OK && a.weights) {
        const int chunks = ceil_div(a.N, 64);
        rc = launch_dependent(kv4_weights_kernel, dim3(chunks < 65535 ? chunks : 65535, a.l.H, a.t.B < 65535 ? a.t.B : 65535), dim3(256), 0, st, a);
    }
    return rc;
}

}  // namespace
}  // namespace bs

using namespace bs;

extern "C" size_t bs_kv4_attend_workspace_bytes(const bs_kv4_cache* cache, int B, int T, int q_heads, int starts, int width, int N)
{
    Kv4 l;
    Plan p;
    const int sms = device_sm_count();
    if (!cache || B <= 0 || T < 0 || N < 0 || q_heads <= 0 || width <= 0 || !kv4_layout(*cache, l) || q_heads % l.H != 0 || sms <= 0 || !plan(l, B, T, q_heads, starts != 0, width, N, sms, p)) return 0;
    return p.bytes();
}

extern "C" int bs_kv4_attend(const void* q, long long q_token, long long q_head, int T, int q_heads, const bs_kv4_cache* cache, const int32_t* table, long long table_pitch, int width,
                             int B, const int32_t* lengths, const int32_t* starts, float scale, void* out, float* weights, long long weights_sequence, long long weights_head, int N,
                             void* workspace, size_t workspace_bytes, void* stream)
{
    Attend a{};
    if (!q || !cache || !cache->data || !table || !lengths || !out || T < 0 || B <= 0 || width <= 0 || (table_pitch != 0 && table_pitch < width) || q_token < 0 || q_head < 0) return BS_ERR_INVALID_ARG;
    if (cache->type != BS_F16 && cache->type != BS_BF16) return BS_ERR_INVALID_ARG;
    if (cache->pages <= 0 || cache->heads <= 0 || cache->D <= 0 || cache->page <= 0 || cache->group <= 0 || q_heads <= 0 || q_heads % cache->heads != 0) return BS_ERR_INVALID_ARG;
    if (!(scale > 0.f) || !(scale * 1.4426950408889634f < INFINITY) || (!starts && T != B)) return BS_ERR_INVALID_ARG;
    if (weights && (N <= 0 || weights_head < N || weights_sequence < 0)) return BS_ERR_INVALID_ARG;
    // rows that several CTAs add to: heads of a sequence side by side, or sequences of a head
    if (weights && B > 1 && weights_sequence < (cache->heads - 1) * weights_head + N && (cache->heads == 1 || weights_sequence < N || weights_head < (B - 1) * weights_sequence + N)) return BS_ERR_INVALID_ARG;
    if (!kv4_layout(*cache, a.l) || q_heads > 65535 || (weights && N > MOST_ROWS)) return BS_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(cache->data) || !aligned16(out) || !aligned16(workspace) || (q_token | q_head) % 8 != 0) return BS_ERR_ALIGNMENT;
    if (T == 0) return BS_OK;
    const int sms = device_sm_count();
    a.status = status_device_ptr();
    if (sms <= 0 || !a.status) return BS_ERR_CUDA;
    Plan p;
    if (!plan(a.l, B, T, q_heads, starts != nullptr, width, weights ? N : 0, sms, p)) return BS_ERR_UNSUPPORTED;
    if (p.bytes() > 0 && (!workspace || workspace_bytes < p.bytes())) return BS_ERR_INVALID_ARG;
    a.t = {table, table_pitch, width, B};
    a.lengths = lengths; a.starts = starts;
    a.q = q; a.q_token = q_token; a.q_head = q_head;
    a.T = T; a.Hq = q_heads; a.per = q_heads / a.l.H;
    a.d_per = make_div(a.per);
    a.d_heads = make_div(a.l.H);
    a.scale = scale * 1.4426950408889634f;
    a.out = out;
    char* ws = static_cast<char*>(workspace);
    if (p.join) {
        a.part = reinterpret_cast<float*>(ws);
        a.stat = reinterpret_cast<float2*>(ws + p.part);
        a.info = reinterpret_cast<int4*>(ws + p.part + p.stat);
        ws += p.part + p.stat + p.info;
    }
    if (weights) {
        a.lse = reinterpret_cast<float*>(ws);
        a.scores = reinterpret_cast<float*>(ws += p.lse);
        a.weights = weights; a.w_sequence = weights_sequence; a.w_head = weights_head; a.N = N;
    }
    a.slots = p.slots;
    return cache->type == BS_F16 ? launch_form<true>(a, p, static_cast<cudaStream_t>(stream)) : launch_form<false>(a, p, static_cast<cudaStream_t>(stream));
}
