// Attention of whole prompts over 16-bit keys and values, packed, causal or not, with heads of queries that share keys: o = softmax(scale q k^T) v on tcgen05.
//
// A tile is 128 rows of queries, row r of it token r / G and head r % G of the G that share a head of keys, so that short prompts fill tiles too.  A CTA, one
// per SM, takes two neighbouring tiles over the same keys, 128 at a time from the last ones that either sees: scores of both in tensor memory (a row a
// lane), two groups of four warps that turn a row's scores into weights, a row a thread, and write them over the scores as 16-bit operands of the
// second product, whose sums stay in tensor memory as well.  While one tile's weights are made the tensor core works for the other.
//
// CTAs go through such pairs, the longest ones first and back and forth, so that all end at about the same time; copies and the first scores of a pair
// begin while the outputs of the one before leave.  Prompts so short that pairs would leave half of the SMs without work take a tile a CTA.
//
// Weights are relative to a maximum that is replaced only when the row's has grown by more than 2^8: sums then have room for it in 32 bits, and the outputs
// are seldom rescaled.  Scores, maxima, sums and outputs have 32 bits; weights are rounded to the type of the values, which is what multiplies them.
//
// 16384 tokens, 32 heads over 8 of 128 channels, causal: 1970 us, 1.12 PFLOP/s, at the power limit (990 W, 1640 MHz); without the weights' work 1590, without loads as well
// 1480.  A tile's weights take 1700 cycles, its products 1050, and 3300 pass for both tiles and 128 keys.  Twelve prompts of up to 4096 tokens 549 us, 500 tokens 13.7.
#include <cuda.h>

#include <mutex>

#include "kv4.h"
#include "mma_kernel.cuh"
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int ROWS = 128, KEYS = 128;
// Warps that make weights, with most of the registers, and four others: one copies, one issues MMAs, one looks for work.  384 threads of 168 registers become 256 of
// 216 and 128 of 72; 72 bytes of a thread go to memory.
constexpr int RING = 4;             // tiles of keys or values on their way; with three the long prompt takes 5 % more
constexpr int SOFTMAX = 8, COPY = SOFTMAX, ISSUE = SOFTMAX + 1, FIND = SOFTMAX + 2, THREADS = (SOFTMAX + 4) * 32;

struct Prompt {
    const int32_t* starts;      // null: one sequence of all rows
    const int32_t* starts_k;
    int B, T, Tk, Hq, H, D, G;
    int tokens, tiles;          // of a tile; of a CTA's piece of work
    int causal;
    float scale;                // times log2(e)
    void* out;                  // [T][Hq][D]
    int* status;
};

// What a CTA does at a time: two tiles of a sequence and head.
struct Work {
    int q0, nq, k0, nk;         // rows of the sequence
    int h, token;               // first token of the first tile
    int blocks[2];              // of keys that a tile sees, 0 without rows
    int any;                    // 0: no more work
};

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// A value that all lanes have, in a register of the warp, where loops over it stay as well.
__device__ __forceinline__ int uniform(int v) { return __reduce_max_sync(0xffffffffu, v); }
struct Rows { int q0, nq, k0, nk, pieces; };
__device__ __forceinline__ Rows rows_of(const Prompt& a, const int32_t* starts, const int32_t* starts_k, int b)
{
    Rows s{0, 0, 0, 0, 0};
    if (b >= a.B) return s;
    s.nq = a.T;
    s.nk = a.Tk;
    if (starts) {
        s.q0 = min(max(starts[b], 0), a.T);
        s.nq = min(max(starts[b + 1], s.q0), a.T) - s.q0;
        s.k0 = min(max(starts_k[b], 0), a.Tk);
        s.nk = min(max(starts_k[b + 1], s.k0), a.Tk) - s.k0;
    }
    s.pieces = (s.nq + a.tiles * a.tokens - 1) / (a.tiles * a.tokens);
    return s;
}
// Blocks of keys that the tokens before `end` of a sequence see.
__device__ __forceinline__ int blocks_of(const Prompt& a, const Rows& s, int end)
{
    const int seen = a.causal ? s.nk - s.nq + min(end, s.nq) : s.nk;
    return seen <= 0 ? 0 : (seen + KEYS - 1) / KEYS;
}
// Pieces of a sequence that see w blocks or more: its last ones.
__device__ __forceinline__ int pieces_from(const Prompt& a, const Rows& s, int w)
{
    if (w <= 0) return s.pieces;
    if (!a.causal) return blocks_of(a, s, 0) >= w ? s.pieces : 0;
    const int step = a.tiles * a.tokens, before = (w - 1) * KEYS - (s.nk - s.nq);      // tokens that see fewer
    return before >= s.nq ? 0 : before < 0 ? s.pieces : s.pieces - before / step;
}
__device__ __forceinline__ int sum_of(int v) { return __reduce_add_sync(0xffffffffu, v); }
__device__ __forceinline__ int up_to_lane(int v)
{
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int u = __shfl_up_sync(0xffffffffu, v, d);
        if ((threadIdx.x & 31) >= d) v += u;
    }
    return v;
}
// The n-th piece of all sequences.  By one warp.  Up to 32 sequences (`mine`: the lane's): those with most blocks first (12 prompts of up to 2000 tokens 159 us, in their
// order 173; 32 of up to 32 tokens 16.3 and 14.1).  More: sequences in their order, a sequence's last pieces first, found by going through them from the first on: 256 of
// up to 64 tokens take 84 us, 1000 of up to 32 tokens 465.
__device__ __forceinline__ bool find(const Prompt& a, const int32_t* starts, const int32_t* starts_k, const Rows& mine, int longest, int n, Work& w)
{
    const int lane = threadIdx.x & 31;
    Rows s = mine;
    int count = s.pieces, behind = 0, before = 0;       // pieces of the lane's sequence that may be the one, how many of its pieces come behind them; pieces in front
    if (a.B <= 32) {
        int lo = 0, hi = longest + 1;                   // more than n pieces see lo blocks or more, but not hi
        if (sum_of(mine.pieces) <= n) return false;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (sum_of(pieces_from(a, mine, mid)) > n) lo = mid;
            else hi = mid;
        }
        behind = pieces_from(a, mine, hi);
        before = sum_of(behind);
        count = pieces_from(a, mine, lo) - behind;
    }
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        if (a.B > 32) {
            s = rows_of(a, starts, starts_k, b0 + lane);
            count = s.pieces;
        }
        const int sum = up_to_lane(count), from = before + sum - count;
        const unsigned here = __ballot_sync(0xffffffffu, n >= from && n < from + count);
        if (here) {
            const int piece = s.pieces - 1 - behind - (n - from);
            w.q0 = s.q0; w.nq = s.nq; w.k0 = s.k0; w.nk = s.nk;
            w.token = piece * a.tiles * a.tokens;
#pragma unroll
            for (int t = 0; t < 2; ++t) w.blocks[t] = t < a.tiles && w.token + t * a.tokens < s.nq ? blocks_of(a, s, w.token + (t + 1) * a.tokens) : 0;
            int* v = &w.q0;
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(Work) / 4); ++i) v[i] = __shfl_sync(0xffffffffu, v[i], __ffs(here) - 1);
            return true;
        }
        before += __shfl_sync(0xffffffffu, sum, 31);
    }
    return false;
}

// D [128 x n] = A (shared memory) B^T (shared memory): 64 channels, rows of 128 bytes, swizzled: four steps of 32 bytes, under one elect in one statement.
#define PROMPT_SS(P) "@p tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, " P ";\n\t"
#define PROMPT_NEXT "add.s64 a, a, 2;\n\tadd.s64 b, b, 2;\n\t"
__device__ __forceinline__ void mma_scores(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 q, %4, 0;\n\tmov.b64 a, %1;\n\tmov.b64 b, %2;\n\telect.sync _|p, 0xffffffff;\n\t"
        PROMPT_SS("q") PROMPT_NEXT PROMPT_SS("1") PROMPT_NEXT PROMPT_SS("1") PROMPT_NEXT PROMPT_SS("1") "}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// D [128 x n] (+)= A (tensor memory) B (shared memory, channels side by side): 64 keys, four steps of 16.
#define PROMPT_TS(P) "@p tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, " P ";\n\t"
#define PROMPT_STEP "add.u32 a, a, 8;\n\tadd.s64 b, b, 128;\n\t" PROMPT_TS("1")
__device__ __forceinline__ void mma_values(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b32 a;\n\t.reg .b64 b;\n\t"
        "setp.ne.b32 q, %4, 0;\n\tmov.b32 a, %1;\n\tmov.b64 b, %2;\n\telect.sync _|p, 0xffffffff;\n\t"
        PROMPT_TS("q") PROMPT_STEP PROMPT_STEP PROMPT_STEP "}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}

// HALVES: of 64 channels.  Tensor memory: scores (and weights over them) of both tiles, outputs of both.
template <bool F16, int HALVES>
__global__ void __launch_bounds__(THREADS, 1) prompt_attend_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv, const __grid_constant__ CUtensorMap to,
                                                                   const __grid_constant__ Prompt a)
{
    typedef W4Type<F16> Ty;
    constexpr int HALF = ROWS * 128, TILE = HALVES * HALF, N = HALVES * 64;
    extern __shared__ unsigned char raw[];
    // queries of the tiles, the ring of keys and values, and outputs of 64 channels of each tile, all in rows of 128 bytes swizzled by address: from a multiple of 1024 on
    unsigned char* smem = raw + (1024 - (smem_u32(raw) & 1023) & 1023);
    __shared__ uint64_t q_full, q_empty, full[RING], empty[RING], s_full[2], p_half[2], p_full[2], o_full[2], work_full[2], work_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ Work works[2];
    __shared__ int4 held_work[SOFTMAX];        // first row of the tile, rows of the sequence from there on, first head
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (warp == COPY) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        mm_fence_before();
    } else if (warp == 0 && lane == 0) {
        mbar_init(&q_full, 1); mbar_init(&q_empty, 1);
        for (int s = 0; s < RING; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&s_full[t], 1); mbar_init(&p_half[t], 4); mbar_init(&p_full[t], 4); mbar_init(&o_full[t], 1);
            mbar_init(&work_full[t], 1); mbar_init(&work_empty[t], SOFTMAX + 2);
        }
        fence_barrier_init();
        fence_proxy_async();
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tq)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tk)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tv)) : "memory");
    }
    __syncthreads();
    mm_fence_after();
    const uint32_t tmem = tmem_slot;
    dependent_begin(a.out);
    bool late = false;
    auto wait = [&](uint64_t* bar, unsigned parity) {
        if (!late && !mm_wait(bar, parity)) {
            late = true;
            atomicOr(a.status, STATUS_TIMEOUT);
        }
    };
    // the next piece of work, for every warp but the one that finds it; false: there is none.  After a wait that ran out there is none either.
    int turn = 0;
    auto take = [&](Work& w) {
        wait(&work_full[turn & 1], turn >> 1 & 1);
        w = works[turn & 1];
        __syncwarp();
        if (lane == 0) mm_arrive(&work_empty[turn & 1]);
        ++turn;
        return !__any_sync(0xffffffffu, late || !w.any);
    };
    if (warp >= SOFTMAX) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;" ::: "memory");
        if (warp == FIND) {
            const int32_t *starts = a.starts ? behind_wait<int32_t>(a.starts) : nullptr, *starts_k = a.starts ? behind_wait<int32_t>(a.starts_k) : nullptr;
            const Rows mine = rows_of(a, starts, starts_k, lane);
            const int longest = uniform(blocks_of(a, mine, mine.nq));
            for (int k = 0, go = 1; go && !late; ++k) {
                // back and forth: who had the longest piece of a round has the shortest of the next
                const int at = k & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
                const long long item = static_cast<long long>(k) * gridDim.x + at;
                Work w{};
                w.any = item < 0x7fffffff && find(a, starts, starts_k, mine, longest, static_cast<int>(item / a.H), w);
                w.h = static_cast<int>(item % a.H);
                go = w.any;
                wait(&work_empty[k & 1], k >> 1 & 1 ^ 1);
                if (lane == 0) {
                    works[k & 1] = w;
                    mm_arrive(&work_full[k & 1]);
                }
                __syncwarp();
            }
        } else if (warp == COPY) {
            Work w;
            unsigned limit = 1u << 20, phase = 1, q_phase = 1;
            int at = 0, issued = 0;
            while (take(w)) {
                const int most = uniform(max(w.blocks[0], w.blocks[1])), h = uniform(w.h), k0 = uniform(w.k0), q0 = uniform(w.q0 + w.token);
                if (most == 0) continue;
                mm_wait_uniform(&q_empty, q_phase, limit);
                q_phase ^= 1;
                if (mm_elect()) {
                    const int bytes = 128 * a.G * a.tokens;        // rows that no tile has keep what the memory holds: they meet nothing
                    mbar_expect_tx(&q_full, a.tiles * HALVES * bytes);
                    for (int t = 0; t < a.tiles; ++t)
                        for (int i = 0; i < HALVES; ++i) tma_load_3d(smem + t * TILE + i * HALF, &tq, &q_full, 64 * i, h * a.G, q0 + t * a.tokens);
                }
                for (int j = 2 * most - 1; j >= 0; --j) {           // keys, then values, of each block
                    mm_wait_uniform(&empty[at], phase, limit);
                    if (mm_elect()) {
                        unsigned char* to = smem + (2 + at) * TILE;
                        mbar_expect_tx(&full[at], TILE);
                        for (int i = 0; i < HALVES; ++i) tma_load_3d(to + i * HALF, j & 1 ? &tk : &tv, &full[at], 64 * i, h, k0 + (j >> 1) * KEYS);
                    }
                    if (++at == RING) { at = 0; phase ^= 1; }
                    ++issued;
                }
            }
            if (limit == 1 && lane == 0) atomicOr(a.status, STATUS_TIMEOUT);
            // no copy outlives the CTA, whatever else was waited for
            limit = 1u << 20;
            if (issued > 0) mm_wait_uniform(&q_full, q_phase, limit);
            for (int i = 0; i < RING && i < issued; ++i) {
                at = at == 0 ? RING - 1 : at - 1;
                if (at == RING - 1) phase ^= 1;
                mm_wait_uniform(&full[at], phase ^ 1, limit);
            }
        } else if (warp == ISSUE) {
            Work w;
            unsigned limit = 1u << 20;
            const uint32_t type = F16 ? 0u : (1u << 7) | (1u << 10);
            const uint32_t score_desc = (1u << 4) | type | (KEYS >> 3) << 17 | (ROWS >> 4) << 24;
            const uint32_t value_desc = (1u << 4) | type | (1u << 16) | (N >> 3) << 17 | (ROWS >> 4) << 24;      // B with its columns side by side
            const uint32_t base = (smem_u32(smem) & 0x3ffff) >> 4;
            // rows of 128 bytes, swizzled in groups of eight: 1024 bytes from group to group; of the values, whose rows are the reduction, HALF from 64 channels to the next
            const uint64_t major = static_cast<uint64_t>(64u | (1u << 14) | (2u << 29)) << 32;
            auto scores = [&](int t, int stage) {
#pragma unroll
                for (int i = 0; i < HALVES; ++i)
                    mma_scores(tmem + t * 128, major | 1u << 16 | (base + (t * TILE + i * HALF) / 16), major | 1u << 16 | (base + ((2 + stage) * TILE + i * HALF) / 16), score_desc, i);
                mm_commit(&s_full[t]);
            };
            int at = 0;
            unsigned phase = 0, q_phase = 0, p_phase[2] = {0, 0}, o_phase[2] = {0, 0};
            auto next = [&] { if (++at == RING) { at = 0; phase ^= 1; } };
            while (take(w)) {
                const int n0 = uniform(w.blocks[0]), n1 = uniform(w.blocks[1]), most = max(n0, n1), nk = uniform(w.nk);
                auto blocks_in = [&](int t) { return t == 0 ? n0 : n1; };
                if (most == 0) continue;
                mm_wait_uniform(&q_full, q_phase, limit);
                q_phase ^= 1;
                mm_wait_uniform(&full[at], phase, limit);
                mm_fence_after();
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (most - 1 < blocks_in(t)) scores(t, at);
                mm_commit(&empty[at]);
                next();
                for (int j = most - 1; j >= 0; --j) {
                    const int v = at;
                    mm_wait_uniform(&full[v], phase, limit);
                    const int left = nk - j * KEYS;
                    if (left < KEYS) {      // rows behind the sequence's last one may hold anything, which zero weights would not keep out
                        for (int i = left * 128 + lane * 16; i < HALF; i += 512)
#pragma unroll
                            for (int k = 0; k < HALVES; ++k) *reinterpret_cast<uint4*>(smem + (2 + v) * TILE + k * HALF + i) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async();
                        __syncwarp();
                    }
                    next();
                    const int k = at;
                    if (j > 0) mm_wait_uniform(&full[k], phase, limit);
                    else mm_commit(&q_empty);               // all scores are on their way
                    const uint64_t values = major | static_cast<uint64_t>(HALF / 16) << 16 | (base + (2 + v) * TILE / 16);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (j < blocks_in(t)) {             // the first 64 keys' weights, then the others'
                            mm_wait_uniform(&p_half[t], p_phase[t], limit);
                            mm_fence_after();
                            mma_values(tmem + 256 + t * 128, tmem + t * 128, values, value_desc, j != blocks_in(t) - 1);
                            mm_wait_uniform(&p_full[t], p_phase[t], limit);
                            mm_fence_after();
                            mma_values(tmem + 256 + t * 128, tmem + t * 128 + 32, values + 512, value_desc, 1);
                            p_phase[t] ^= 1;
                            if (j == 0) {
                                mm_commit(&o_full[t]);
                                o_phase[t] ^= 1;
                            }
                        }
                        if (j > 0 && j - 1 < blocks_in(t)) scores(t, k);
                    }
                    mm_commit(&empty[v]);
                    if (j > 0) {
                        mm_commit(&empty[k]);
                        next();
                    }
                }
            }
            if (limit == 1 && lane == 0) atomicOr(a.status, STATUS_TIMEOUT);
            limit = 1u << 20;           // nor do the MMAs outlive the tensor memory
#pragma unroll
            for (int t = 0; t < 2; ++t) mm_wait_uniform(&o_full[t], o_phase[t] ^ 1, limit);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;" ::: "memory");
        const int t = warp >> 2, row = (warp & 3) * 32 + lane, row_token = row / a.G, row_head = row - row_token * a.G;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16, s_at = tmem + t * 128 + lanes, o_at = tmem + 256 + t * 128 + lanes;
        const u64 scale2 = f2_pack(__float_as_uint(a.scale), __float_as_uint(a.scale));
        unsigned char* held = smem + (2 + RING) * TILE + t * HALF;
        unsigned s_phase = 0, o_phase = 0;
        Work w;
        while (take(w)) {
            const int blocks = t == 0 ? w.blocks[0] : w.blocks[1];
            const int first = w.token + t * a.tokens, token = first + row_token;
            const int seen = a.causal ? min(w.nk - w.nq + token + 1, w.nk) : w.nk;                 // keys that the row sees
            const int all = a.causal ? min(w.nk - w.nq + first + 1, w.nk) : w.nk;                  // and that all rows of the tile see
            // what the outputs need waits in memory: the registers are the scores'
            if (lane == 0) held_work[warp] = make_int4(w.q0 + first, w.nq - first, w.h * a.G, 0);
            __syncwarp();
            float top = -INFINITY, total = 0.f;
            for (int j = blocks - 1; j >= 0; --j) {
                wait(&s_full[t], s_phase);
                s_phase ^= 1;
                mm_fence_after();
                uint32_t v[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) mm_ld32(s_at + 32 * i, v[i]);
                mm_ld_wait();
#pragma unroll
                for (int i = 0; i < 4; ++i) mm_landed(v[i]);
                if ((j + 1) * KEYS > all) {
                    const int left = seen - j * KEYS;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int l = left - 32 * i;
                        const uint32_t m = l >= 32 ? 0xffffffffu : l <= 0 ? 0u : (1u << l) - 1;
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[i][k] = m >> k & 1 ? v[i][k] : 0xff800000u;
                    }
                }
                float high[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t* x = &v[i / 2][i % 2 * 16];
                    high[i] = max3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]));
#pragma unroll
                    for (int k = 3; k < 15; k += 2) high[i] = max3(high[i], __uint_as_float(x[k]), __uint_as_float(x[k + 1]));
                    high[i] = fmaxf(high[i], __uint_as_float(x[15]));
                }
                const float now = fmaxf(max3(max3(high[0], high[1], high[2]), high[3], high[4]), max3(high[5], high[6], high[7]));
                const bool grown = (now - top) * a.scale > 8.f || (top == -INFINITY && now > -INFINITY);
                if (__any_sync(0xffffffffu, grown)) {
                    const float to = grown ? now : top, f = grown ? exp2_of((top - to) * a.scale) : 1.f;
                    top = to;
                    total *= f;
                    if (j != blocks - 1) {      // the outputs so far: the scores' barrier says that their last product is done
#pragma unroll
                        for (int i = 0; i < N; i += 32) {
                            uint32_t o[32];
                            mm_ld32(o_at + i, o);
                            mm_ld_wait();
                            mm_landed(o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            mm_st16(o_at + i, o);
                            mm_st16(o_at + i + 16, o + 16);
                        }
                    }
                }
                // weights of up to 2^8 are times 2^7 where fp16 holds them, which leaves bits to those down to 2^-32 of the largest one
                const float lift = F16 ? 7.f : 0.f;
                float base_of = top == -INFINITY ? 0.f : fmaf(-top, a.scale, lift);
                if (__any_sync(0xffffffffu, fabsf(base_of) >= 0x1p20f)) {           // its last place would be an eighth and more: distances first
                    const float less = top == -INFINITY ? 0.f : top;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[i][k] = __float_as_uint(__uint_as_float(v[i][k]) - less);
                    base_of = lift;
                }
                const u64 base2 = f2_pack(__float_as_uint(base_of), __float_as_uint(base_of));
                u64 sums[4] = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t p[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        uint32_t lo, hi;
                        f2_split(f2_fma(f2_pack(v[i][2 * k], v[i][2 * k + 1]), scale2, base2), lo, hi);
                        const float x = exp2_of(__uint_as_float(lo)), y = exp2_of(__uint_as_float(hi));
                        sums[k & 3] = f2_add(sums[k & 3], f2_pack(__float_as_uint(x), __float_as_uint(y)));
                        p[k] = Ty::round2(x, y);
                    }
                    mm_st16(s_at + 16 * i, p);
                    if (i & 1) {
                        mm_st_wait();
                        mm_fence_before();
                        __syncwarp();
                        if (lane == 0) mm_arrive(i == 1 ? &p_half[t] : &p_full[t]);
                    }
                }
                uint32_t lo, hi;
                f2_split(f2_add(f2_add(sums[0], sums[1]), f2_add(sums[2], sums[3])), lo, hi);
                total += __uint_as_float(lo) + __uint_as_float(hi);
            }
            if (blocks > 0) {
                wait(&o_full[t], o_phase);
                o_phase ^= 1;
                mm_fence_after();
            }
            const float inverse = total == 0.f ? 0.f : 1.f / total;
            const int4 place = held_work[warp];
            const bool box = t < a.tiles && a.tokens <= place.y;          // all of the tile's rows are there: they leave as boxes of 64 channels
            uint16_t* out = nullptr;
            if (row < a.tokens * a.G && t < a.tiles && row_token < place.y)
                out = static_cast<uint16_t*>(a.out) + (static_cast<long long>(place.x + row_token) * a.Hq + place.z + row_head) * a.D;
#pragma unroll
            for (int i = 0; i < HALVES; ++i) {
                if (box) {
                    if (row == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");          // the box before has been read
                    asm volatile("bar.sync %0, 128;" ::"r"(1 + t) : "memory");
                }
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    uint32_t o[32];
                    if (blocks > 0) {
                        mm_ld32(o_at + 64 * i + 32 * n, o);
                        mm_ld_wait();
                        mm_landed(o);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t p[4];
#pragma unroll
                        for (int m = 0; m < 4; ++m)
                            p[m] = total == 0.f ? 0u : Ty::round2(__uint_as_float(o[8 * k + 2 * m]) * inverse, __uint_as_float(o[8 * k + 2 * m + 1]) * inverse);
                        if (box) *reinterpret_cast<uint4*>(held + row * 128 + ((4 * n + k ^ (row & 7)) * 16)) = make_uint4(p[0], p[1], p[2], p[3]);
                        else if (out && 64 * i + 32 * n + 8 * k < a.D) *reinterpret_cast<uint4*>(out + 64 * i + 32 * n + 8 * k) = make_uint4(p[0], p[1], p[2], p[3]);
                    }
                }
                if (box) {
                    fence_proxy_async();
                    asm volatile("bar.sync %0, 128;" ::"r"(1 + t) : "memory");
                    if (row == 0) {
                        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                                     ::"l"(reinterpret_cast<uint64_t>(&to)), "r"(smem_u32(held)), "r"(64 * i), "r"(place.z), "r"(place.x) : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                }
            }
            mm_fence_before();          // the next piece's first product may write over them once its weights are there
        }
        if (row == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    }
    __syncthreads();
    if (warp == COPY) {
        mm_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn()
{
    static EncodeFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* q = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &q, cudaEnableDefault, &r) == cudaSuccess && r == cudaDriverEntryPointSuccess) fn = reinterpret_cast<EncodeFn>(q);
    });
    return fn;
}
// Vectors [n][heads][D], fetched in boxes of 64 channels, `wide` heads and `high` rows.  A single row or head may be any distance from the next.
bool encode(CUtensorMap* tm, const void* p, bool f16, int n, int heads, int D, long long token, long long head, int wide, int high)
{
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(n)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(heads == 1 ? D : head) * 2, static_cast<cuuint64_t>(n == 1 ? static_cast<long long>(D) * heads : token) * 2};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(wide), static_cast<cuuint32_t>(high)}, es[3] = {1, 1, 1};
    return fn(tm, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool F16, int HALVES>
int launch(const CUtensorMap (&maps)[4], const Prompt& a, long long ctas, cudaStream_t st)
{
    constexpr int smem = 1024 + ((2 + RING) * HALVES + 2) * ROWS * 128;
    if (!allow_shared<prompt_attend_kernel<F16, HALVES>>(smem)) return BS_ERR_CUDA;
    return launch_dependent(prompt_attend_kernel<F16, HALVES>, dim3(static_cast<unsigned>(ctas)), dim3(THREADS), smem, st, maps[0], maps[1], maps[2], maps[3], a);
}

}  // namespace
}  // namespace bs

using namespace bs;

extern "C" int bs_attend_prompt(const void* q, long long q_token, long long q_head, int T, int q_heads, const void* k, long long k_token, long long k_head, const void* v,
                                long long v_token, long long v_head, int Tk, int heads, int D, bs_float_t type, int B, const int32_t* starts, const int32_t* starts_k, float scale, int causal,
                                void* out, void* stream)
{
    if (!q || !k || !v || !out || T < 0 || Tk < 0 || q_heads <= 0 || heads <= 0 || D <= 0 || q_heads % heads != 0 || B <= 0) return BS_ERR_INVALID_ARG;
    if ((type != BS_F16 && type != BS_BF16) || !(scale > 0.f) || !(scale * 1.4426950408889634f < INFINITY)) return BS_ERR_INVALID_ARG;
    if (q_token < 0 || q_head < 0 || k_token < 0 || k_head < 0 || v_token < 0 || v_head < 0) return BS_ERR_INVALID_ARG;
    if ((starts == nullptr) != (starts_k == nullptr) || (!starts && B != 1)) return BS_ERR_INVALID_ARG;
    Prompt a{};
    a.G = q_heads / heads;
    if (D > 128 || D % 8 != 0 || a.G > ROWS || T > MOST_ROWS || Tk > MOST_ROWS) return BS_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || (q_token | q_head | k_token | k_head | v_token | v_head) % 8 != 0) return BS_ERR_ALIGNMENT;
    if (T == 0) return BS_OK;
    a.starts = starts; a.starts_k = starts_k;
    a.B = B; a.T = T; a.Tk = Tk; a.Hq = q_heads; a.H = heads; a.D = D;
    a.tokens = ROWS / a.G;
    a.causal = causal != 0;
    a.scale = scale * 1.4426950408889634f;
    a.out = out;
    a.status = status_device_ptr();
    if (!a.status) return BS_ERR_CUDA;
    const int sms = device_sm_count();
    if (sms <= 0) return BS_ERR_CUDA;
    // pieces of two tiles, or of one while there are SMs for all of them (500 tokens: 14.3 us with two)
    const long long singles = (ceil_div_ll(T, a.tokens) + (B - 1)) * heads, pairs = (ceil_div_ll(T, 2 * a.tokens) + (B - 1)) * heads;
    a.tiles = singles <= sms ? 1 : 2;
    const long long pieces = a.tiles == 1 ? singles : pairs, ctas = pieces < sms ? pieces : sms;
    if (pieces > 0x7fff0000) return BS_ERR_UNSUPPORTED;
    const bool f16 = type == BS_F16;
    CUtensorMap maps[4];            // queries, keys, values, outputs
    // without keys nothing is fetched; a map has to have rows all the same
    const int rows_k = Tk > 0 ? Tk : 1, heads_k = Tk > 0 ? heads : 1;
    if (!encode(&maps[0], q, f16, T, q_heads, D, q_token, q_head, a.G, a.tokens) || !encode(&maps[1], k, f16, rows_k, heads_k, D, k_token, k_head, 1, KEYS) ||
        !encode(&maps[2], v, f16, rows_k, heads_k, D, v_token, v_head, 1, KEYS) ||
        !encode(&maps[3], out, f16, T, q_heads, D, static_cast<long long>(q_heads) * D, D, a.G, a.tokens))
        return BS_ERR_UNSUPPORTED;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (D <= 64) return f16 ? launch<true, 1>(maps, a, ctas, st) : launch<false, 1>(maps, a, ctas, st);
    return f16 ? launch<true, 2>(maps, a, ctas, st) : launch<false, 2>(maps, a, ctas, st);
}
