// Product of many rows of x with 4-bit weights on tcgen05.mma: the weights are the A operand, 128 rows a tile, expanded to 16 bits in tensor memory; x is B.
//
// The codes less their zero points are exact in 16 bits and the scales are not folded into them: a group's sums of exact products come out of the tensor
// core in an accumulator of their own, and warps with the running totals in registers take them over, scaled in 32 bits, while the next group is
// multiplied.  Folding the scale in would round every weight and double the error of the result.
//
// Roles of a CTA, one per SM: tensor copies of x and of the weights' blocks, MMA issue, warps that expand a row a thread into tensor memory, warps that scale
// and add.  A step is 128 columns.  The MMA warp's waits and commits, 100 to 160 cycles each, would cost more than the 512 cycles of a step's MMAs:
// whatever a step needs (x, its expanded weights, and with one group a step a free accumulator) arrives at one barrier, and one commit frees
// all of it again.
//
// 4096 x 16384 x 4096: 680 us, 810 TFLOP/s (half of what the tensor core does; 585 us in a short run, before the power limit is met): a step takes about
// 1100 cycles, the 512 of its MMAs beside 750 in which an accumulator is read out, which the other two hide only in part, and hand-offs.  200 x 4096 x
// 4096: 19.9 us, of which 4 are MMAs: the first blocks' way in, 14 steps a CTA, the parts' way through memory and the second launch.
//
// Work: tiles of 128 rows by up to 128 rows of x.  A CTA takes whole tiles, neighbours at a time, as long as every CTA gets one; what is left, less than
// two tiles a CTA, is cut (unless that saves little) into equal runs of (tile, 128 columns), and a small kernel adds the parts of the tiles that were cut, in
// their order.
#include <cuda.h>

#include <mutex>

#include "mma_kernel.cuh"
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int ROWS = 128, BLOCKS = ROWS / W4_ROWS;      // of a tile
constexpr int RING = 4, SCALE_SLOTS = 32;         // stages of x: steps on their way

struct MmaTiles {
    W4Gemm g;
    int n;                      // rows of x in a tile, a multiple of 32
    int mts, ots;               // tiles of x's rows and of the weights' rows
    int waves;                  // whole tiles of every CTA
    int per;                    // steps of 128 columns in a run
    int ctas;
    float* part;                // [2 ctas][n][ROWS]: the parts of the tiles that a run begins and ends in
};

// Tile t: eight tiles of x's rows side by side, then the weights' next rows, so that what runs at the same time shares both.
__device__ __forceinline__ void tile_place(const MmaTiles& a, int t, int& mt, int& ot)
{
    const int wide = 8 * a.ots, group = t / wide, in = t - group * wide, rows = min(8, a.mts - group * 8);
    ot = in / rows;
    mt = group * 8 + in - ot * rows;
}
// A CTA's stretches of work, one after the other: steps [c0, c1) of a tile.
struct Stretch {
    int wave, pos, end;         // whole tiles done; steps of the run
    int tile, c0, c1, part;     // part: where a part of a tile goes, -1: the whole tile is here
    __device__ __forceinline__ Stretch(const MmaTiles& a) : wave(0)
    {
        const long long steps = static_cast<long long>(a.mts) * a.ots * a.g.l.cbs - static_cast<long long>(a.waves) * a.ctas * a.g.l.cbs;
        const long long b = static_cast<long long>(blockIdx.x) * a.per;
        pos = a.per == 0 ? 0 : static_cast<int>(b < steps ? b : steps);
        end = a.per == 0 ? 0 : static_cast<int>(b + a.per < steps ? b + a.per : steps);
        first = pos;
    }
    __device__ __forceinline__ bool next(const MmaTiles& a)
    {
        const int cbs = a.g.l.cbs;
        if (wave < a.waves) {
            tile = wave++ * a.ctas + blockIdx.x;
            c0 = 0; c1 = cbs; part = -1;
            return tile < a.mts * a.ots;
        }
        if (pos >= end) return false;
        tile = pos / cbs;
        c0 = pos - tile * cbs;
        c1 = min(cbs, c0 + end - pos);
        // a run begins in one tile and ends in another: two places; a tile that both begins before and ends behind the run has the first
        part = c0 == 0 && c1 == cbs ? -1 : 2 * static_cast<int>(blockIdx.x) + (pos != first);
        pos += c1 - c0;
        tile += a.waves * a.ctas;
        return true;
    }
    int first;
};

__device__ __forceinline__ void w4_st32(uint32_t taddr, const uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
          "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
          "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}
// D[128 x n] (+)= A (tensor memory) B (shared memory): STEPS times 16 columns of the reduction (8 columns of A, 32 bytes of B's rows each) under one elect, in
// one statement: descriptors that leave it move through vector registers, 90 cycles an MMA.
#define W4_MMA(A, B, P) "@p tcgen05.mma.cta_group::1.kind::f16 [%0], [" A "], " B ", %3, " P ";\n\t"
#define W4_STEP "add.u32 u, u, 8;\n\tadd.s64 t, t, 2;\n\t" W4_MMA("u", "t", "1")
template <int STEPS>
__device__ __forceinline__ void w4_mma(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t acc)
{
    const uint64_t b = (static_cast<uint64_t>(b_hi) << 32) | b_lo;
    if constexpr (STEPS == 4)
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t.reg .b32 u;\n\t.reg .b64 t;\n\t"
            "setp.ne.b32 q, %4, 0;\n\tmov.b32 u, %1;\n\tmov.b64 t, %2;\n\telect.sync _|p, 0xffffffff;\n\t"
            W4_MMA("u", "t", "q") W4_STEP W4_STEP W4_STEP "}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t.reg .b32 u;\n\t.reg .b64 t;\n\t"
            "setp.ne.b32 q, %4, 0;\n\tmov.b32 u, %1;\n\tmov.b64 t, %2;\n\telect.sync _|p, 0xffffffff;\n\t"
            W4_MMA("u", "t", "q") W4_STEP "}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}

// A position in a ring of stages, and the parity of its round.
template <int N>
struct Turn {
    int at;
    unsigned phase;
    __device__ __forceinline__ Turn() : at(0), phase(0) {}
    __device__ __forceinline__ void next() { if (++at == N) { at = 0; phase ^= 1; } }
};

// FEW: up to 64 rows of x, bound by the weights: four warps scale, otherwise eight.  The threads' registers are dealt anew: 640 of 96 become 128 (copies, MMA
// issue) of 40, 256 (expansion) of 96 and 256 (totals) of 120; with few rows 512 of 128 become 128 of 40, 256 of 104 and 128 of 168.
template <bool FEW> struct Roles {
    static constexpr int EXPAND = 8, SCALE = FEW ? 4 : 8, WARPS = 4 + EXPAND + SCALE, W_STAGES = FEW ? 8 : 4;
    static constexpr int N = FEW ? 64 : 128;                    // most rows of x in a tile
    static constexpr int PIECES = N * 4 / SCALE / 16;           // 16 columns each, of a thread's totals
};
// Three accumulators of N columns (reading one takes 750 cycles while the next one's MMAs run: with two the MMAs wait for it), two buffers of 64 of weights.
constexpr int SUMS = 3, TMEM_COLUMNS = 512, TMEM_A = 384;
template <bool MORE, int N> __device__ __forceinline__ void registers()
{
    if (MORE) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

template <bool F16, int NG, bool ZEROS, bool FEW>
__global__ void __launch_bounds__(Roles<FEW>::WARPS * 32, 1) w4_mma_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ CUtensorMap tw, const __grid_constant__ MmaTiles a)
{
    typedef W4Type<F16> Ty;
    typedef typename Ty::T T;
    typedef Roles<FEW> Ro;
    constexpr int ENTRY = ZEROS ? 8 : 4, BLOCK = W4_CODES + NG * 8 * ENTRY, WS = Ro::W_STAGES;
    extern __shared__ unsigned char raw[];
    // x [RING][2][n][128 bytes], swizzled by address: from a multiple of 1024 on; weights [WS][BLOCKS][BLOCK]
    unsigned char* smem = raw + (1024 - (smem_u32(raw) & 1023) & 1023);
    __shared__ uint64_t full[RING], done[RING], w_full[WS], w_empty[WS], d_full[SUMS], d_empty[SUMS];     // the last two where a step has several groups
    __shared__ float scales[SCALE_SLOTS][ROWS];
    __shared__ uint32_t tmem_slot;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const W4Layout& l = a.g.l;
    unsigned char* wsm = smem + static_cast<size_t>(RING) * a.n * 256;
    if (warp == 3) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(TMEM_COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        mm_fence_before();
    } else if (warp == 0 && lane == 0) {
        for (int s = 0; s < RING; ++s) { mbar_init(&full[s], 5 + (NG == 1 ? Ro::SCALE : 0)); mbar_init(&done[s], 1); }
        for (int s = 0; s < WS; ++s) { mbar_init(&w_full[s], 1); mbar_init(&w_empty[s], 4); }
        for (int s = 0; s < SUMS; ++s) { mbar_init(&d_full[s], 1); mbar_init(&d_empty[s], Ro::SCALE); }
        fence_barrier_init();
        fence_proxy_async();
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tx)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tw)) : "memory");
    }
    __syncthreads();
    mm_fence_after();
    const uint32_t tmem = tmem_slot, tmem_a = tmem + TMEM_A;
    dependent_begin(a.g.w);
    bool late = false;          // a wait ran out: later ones are not waited for
    auto wait = [&](uint64_t* bar, unsigned parity) {
        if (!late && !mm_wait(bar, parity)) {
            late = true;
            atomicOr(a.g.status, STATUS_TIMEOUT);
        }
    };
    Stretch s(a);
    if (warp < 4) {
        registers<false, 40>();
        if (warp == 0) {
            Turn<RING> x;
            unsigned limit = 1u << 20;
            int issued = 0;
            while (s.next(a)) {
                int mt, ot;
                tile_place(a, s.tile, mt, ot);
                for (int c = s.c0; c < s.c1; ++c) {
                    mm_wait_uniform(&done[x.at], x.phase ^ 1, limit);
                    if (mm_elect()) {
                        unsigned char* to = smem + static_cast<size_t>(x.at) * a.n * 256;
                        mbar_expect_tx(&full[x.at], a.n * 256);
                        tma_load_2d(to, &tx, &full[x.at], c * W4_COLS, mt * a.n);
                        tma_load_2d(to + a.n * 128, &tx, &full[x.at], c * W4_COLS + 64, mt * a.n);
                    }
                    x.next();
                    ++issued;
                }
            }
            if (limit == 1 && lane == 0) atomicOr(a.g.status, STATUS_TIMEOUT);
            limit = 1u << 20;
            for (int i = 0; i < RING && i < issued; ++i) {      // no copy outlives the CTA, whatever else was waited for
                x.at = x.at == 0 ? RING - 1 : x.at - 1;
                if (x.at == RING - 1) x.phase ^= 1;
                mm_wait_uniform(&full[x.at], x.phase, limit);
            }
        } else if (warp == 1) {
            Turn<RING> x;
            Turn<2> ab;
            Turn<SUMS> d;
            unsigned limit = 1u << 20;
            bool any = false;
            const uint32_t base = (smem_u32(smem) & 0x3ffff) >> 4;
            // K-major rows of 128 bytes, swizzled in groups of eight: 1024 bytes from group to group
            const uint32_t b_hi = 64u | (1u << 14) | (2u << 29);
            while (s.next(a)) {
                int mt, ot;
                tile_place(a, s.tile, mt, ot);
                const int m0 = mt * a.n, rows = min(a.n, (a.g.M - m0 + 31) & ~31);
                const uint32_t idesc = (1u << 4) | (F16 ? 0u : (1u << 7) | (1u << 10)) | (static_cast<uint32_t>(rows >> 3) << 17) | (static_cast<uint32_t>(ROWS >> 4) << 24);
                for (int c = s.c0; c < s.c1; ++c) {
                    mm_wait_uniform(&full[x.at], x.phase, limit);
                    mm_fence_after();
                    const uint32_t xs = base + static_cast<uint32_t>(x.at * a.n * 16), as = tmem_a + ab.at * 64;
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        if (NG > 1) {
                            mm_wait_uniform(&d_empty[d.at], d.phase ^ 1, limit);
                            mm_fence_after();
                        }
                        constexpr int STEPS = NG == 4 ? 2 : 4;      // 64 columns of x lie together
#pragma unroll
                        for (int k = 0; k < 8 / NG; k += STEPS) {
                            const int step = g * (8 / NG) + k;
                            const uint32_t b = xs + static_cast<uint32_t>((step >> 2) * a.n * 8 + (step & 3) * 2);
                            w4_mma<STEPS>(tmem + d.at * Ro::N, as + step * 8, (b & 0x3fff) | (1u << 16), b_hi, idesc, k == 0 ? 0u : 1u);
                        }
                        if (NG > 1) mm_commit(&d_full[d.at]);
                        d.next();
                    }
                    mm_commit(&done[x.at]);
                    any = true;
                    x.next();
                    ab.next();
                }
            }
            if (limit == 1 && lane == 0) atomicOr(a.g.status, STATUS_TIMEOUT);
            limit = 1u << 20;           // nor do the MMAs outlive the tensor memory
            if (any) mm_wait_uniform(&done[x.at == 0 ? RING - 1 : x.at - 1], x.at == 0 ? x.phase ^ 1 : x.phase, limit);
        } else if (warp == 2) {
            // the blocks of eight rows of blocks in one copy: as copies of their own they took 130 cycles each to start, twice the time of a step
            Turn<WS> w;
            unsigned limit = 1u << 20;
            int issued = 0;
            while (s.next(a)) {
                int mt, ot;
                tile_place(a, s.tile, mt, ot);
                for (int c = s.c0; c < s.c1; ++c) {
                    mm_wait_uniform(&w_empty[w.at], w.phase ^ 1, limit);
                    if (mm_elect()) {
                        mbar_expect_tx(&w_full[w.at], BLOCKS * BLOCK);
                        tma_load_4d(wsm + w.at * BLOCKS * BLOCK, &tw, &w_full[w.at], 0, c, ot * BLOCKS, 0);
                    }
                    w.next();
                    ++issued;
                }
            }
            if (limit == 1 && lane == 0) atomicOr(a.g.status, STATUS_TIMEOUT);
            limit = 1u << 20;
            for (int i = 0; i < WS && i < issued; ++i) {
                w.at = w.at == 0 ? WS - 1 : w.at - 1;
                if (w.at == WS - 1) w.phase ^= 1;
                mm_wait_uniform(&w_full[w.at], w.phase, limit);
            }
        }
    } else if (warp < 4 + Ro::EXPAND) {
        registers<false, FEW ? 104 : 96>();
        // a thread owns a row of the tile; each team of four warps takes every other step
        const int team = (warp - 4) >> 2, row = (warp & 3) * 32 + lane, r = row & 15;
        const uint32_t mine = smem_u32(wsm) + (row >> 4) * BLOCK, lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        Turn<WS> w;
        Turn<RING> x;
        int round = 0;
        while (s.next(a)) {
            for (int c = s.c0; c < s.c1; ++c) {
                if ((x.at & 1) == team) {
                    wait(&w_full[w.at], w.phase);
                    const uint32_t block = mine + w.at * BLOCKS * BLOCK;
                    uint4 code[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(code[t].x), "=r"(code[t].y), "=r"(code[t].z), "=r"(code[t].w)
                                     : "r"(block + t * 256 + ((r & 8) | ((r & 7) ^ 2 * t)) * 16) : "memory");
                    uint32_t scale[NG], zero[NG];
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const uint32_t e = block + W4_CODES + (g * 8 + (r & 7)) * ENTRY + (r >> 3) * 2;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=r"(scale[g]) : "r"(e) : "memory");
                        zero[g] = 8;
                        if (ZEROS) asm volatile("ld.shared.u16 %0, [%1];" : "=r"(zero[g]) : "r"(e + 4) : "memory");
                    }
                    // the numbers first: the buffer's last MMAs may still run
                    uint32_t v[2][32];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            uint32_t p[4];
                            Ty::pairs(word_of(code[t], j), zero[j * NG / 4] * 0x00010001u, p);
#pragma unroll
                            for (int i = 0; i < 4; ++i) v[j >> 1][16 * (j & 1) + 4 * t + i] = p[i];
                        }
                    wait(&done[x.at ^ 2], x.at < 2 ? x.phase ^ 1 : x.phase);      // the step before the last one
                    mm_fence_after();
                    w4_st32(tmem_a + team * 64 + lanes, v[0]);
                    w4_st32(tmem_a + team * 64 + 32 + lanes, v[1]);
                    // that step is done and all rounds before its last three are scaled: the slots of these are free
#pragma unroll
                    for (int g = 0; g < NG; ++g) scales[(round + g) % SCALE_SLOTS][row] = Ty::lo(scale[g]);
                    mm_st_wait();
                    mm_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        mm_arrive(&full[x.at]);
                        mm_arrive(&w_empty[w.at]);
                    }
                }
                round += NG;
                w.next();
                x.next();
            }
        }
    } else {
        registers<true, FEW ? 168 : 120>();
        // a thread owns a row of the tile and all of its columns, or with eight warps half of them
        const int half = (warp - 4 - Ro::EXPAND) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        Turn<RING> x;           // of the steps, where each is a round
        Turn<SUMS> d;
        int round = 0;
        if (NG == 1 && lane == 0)       // the accumulators of the first steps are free
            for (int i = 0; i < SUMS; ++i) mm_arrive(&full[i]);
        while (s.next(a)) {
            int mt, ot;
            tile_place(a, s.tile, mt, ot);
            const int m0 = mt * a.n, rows = min(a.n, (a.g.M - m0 + 31) & ~31), width = rows * 4 / Ro::SCALE, n0 = half * width;
            u64 tot[Ro::PIECES][8];
#pragma unroll
            for (int p = 0; p < Ro::PIECES; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) tot[p][i] = 0;
            const int rounds = (s.c1 - s.c0) * NG;
            for (int k = 0; k < rounds; ++k) {
                wait(NG == 1 ? &done[x.at] : &d_full[d.at], NG == 1 ? x.phase : d.phase);
                mm_fence_after();
                const uint32_t from = tmem + d.at * Ro::N + n0 + lanes;
                const float sc = scales[round % SCALE_SLOTS][row];
                const u64 ss = f2_pack(__float_as_uint(sc), __float_as_uint(sc));
#pragma unroll
                for (int h = 0; h < Ro::PIECES; h += 2) {
                    uint32_t v[32];
                    if (h * 16 + 32 <= width) mm_ld32(from + h * 16, v);
                    else if (h * 16 < width) mm_ld16(from + h * 16, reinterpret_cast<uint32_t (&)[16]>(v[0]));
                    mm_ld_wait();
                    mm_landed(v);
                    if (h + 2 >= Ro::PIECES) {      // the accumulator is free
                        mm_fence_before();
                        __syncwarp();
                        if (lane == 0) mm_arrive(NG == 1 ? &full[(x.at + SUMS) % RING] : &d_empty[d.at]);
                    }
#pragma unroll
                    for (int p = 0; p < 2; ++p)
                        if ((h + p) * 16 < width) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) tot[h + p][i] = f2_fma(f2_pack(v[16 * p + 2 * i], v[16 * p + 2 * i + 1]), ss, tot[h + p][i]);
                        }
                }
                x.next();
                d.next();
                ++round;
            }
            const int o = ot * ROWS + row, left = a.g.M - m0 - n0;      // rows of x that there are
            if (s.part < 0) {
                const float bias = a.g.bias && o < l.O ? static_cast<float>(static_cast<const T*>(a.g.bias)[o]) : 0.f;
                T* y = static_cast<T*>(a.g.y) + static_cast<long long>(m0 + n0) * a.g.ldy;
                if (width <= left && ot * ROWS + ROWS <= l.O && (a.g.ldy & 1) == 0) {
                    // neighbouring lanes trade: each stores two columns of y in one of two rows
                    y += (lane & 1) * a.g.ldy + (o & ~1);
#pragma unroll
                    for (int p = 0; p < Ro::PIECES; ++p)
                        if (p * 16 < width) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                uint32_t lo, hi;
                                f2_split(tot[p][i], lo, hi);
                                const uint32_t both = Ty::round2(fmaf(__uint_as_float(lo), Ty::PART, bias), fmaf(__uint_as_float(hi), Ty::PART, bias)), other = __shfl_xor_sync(0xffffffffu, both, 1);
                                *reinterpret_cast<uint32_t*>(y) = lane & 1 ? __byte_perm(other, both, 0x7632) : __byte_perm(both, other, 0x5410);
                                y += 2 * a.g.ldy;
                            }
                        }
                } else if (o < l.O) {
                    y += o;
#pragma unroll
                    for (int p = 0; p < Ro::PIECES; ++p)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            uint32_t lo, hi;
                            f2_split(tot[p][i], lo, hi);
                            const int m = p * 16 + 2 * i;
                            if (m < width && m < left) y[m * a.g.ldy] = Ty::round(fmaf(__uint_as_float(lo), Ty::PART, bias));
                            if (m < width && m + 1 < left) y[(m + 1) * a.g.ldy] = Ty::round(fmaf(__uint_as_float(hi), Ty::PART, bias));
                        }
                }
            } else {
                // rows of x that are not there are written too: their places are the tile's
                float* out = a.part + (static_cast<size_t>(s.part) * a.n + n0) * ROWS + row;
#pragma unroll
                for (int p = 0; p < Ro::PIECES; ++p)
                    if (p * 16 < width) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            uint32_t lo, hi;
                            f2_split(tot[p][i], lo, hi);
                            out[(p * 16 + 2 * i) * ROWS] = __uint_as_float(lo) * Ty::PART;
                            out[(p * 16 + 2 * i + 1) * ROWS] = __uint_as_float(hi) * Ty::PART;
                        }
                    }
            }
        }
    }
    mm_fence_before();
    __syncthreads();
    mm_fence_after();
    if (warp == 3) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLUMNS) : "memory");
}

// Adds the parts of the tiles that were cut, in the order of the reduction, from L2; bound by launch and latency, about 3 us.  blockIdx.x: the run whose beginning is the first cut in its tile.  A thread: four
// columns of y in one row.
template <bool F16>
__global__ void __launch_bounds__(256) w4_join_kernel(const __grid_constant__ MmaTiles a)
{
    typedef typename W4Type<F16>::T T;
    const float* part = dependent_begin(a.part);
    const int cbs = a.g.l.cbs, run = blockIdx.x + 1, steps = (a.mts * a.ots - a.waves * a.ctas) * cbs, cut = run * a.per;       // below 2^31, as all steps are
    const int t = cut / cbs, beg = t * cbs;
    if (cut >= steps || cut == beg || cut - a.per > beg) return;       // no cut, or an earlier run's beginning lies in this tile
    const int last = (beg + cbs - 1) / a.per;
    int mt, ot;
    tile_place(a, t + a.waves * a.ctas, mt, ot);
    const int m0 = mt * a.n, i = blockIdx.y * blockDim.x + threadIdx.x, m = i / (ROWS / 4), r = i % (ROWS / 4) * 4, o = ot * ROWS + r;
    if (m >= min(a.n, a.g.M - m0) || o >= a.g.l.O) return;
    // the tile is what run - 1 ends in (or begins in, at the tile's own beginning), and what the others begin in
    const size_t place = static_cast<size_t>(a.n) * ROWS, at = static_cast<size_t>(m) * ROWS + r;
    float4 v = *reinterpret_cast<const float4*>(part + (2 * (run - 1) + (cut - a.per < beg)) * place + at);
#pragma unroll 4
    for (int c = run; c <= last; ++c) {
        const float4 w = *reinterpret_cast<const float4*>(part + 2 * c * place + at);
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
    }
    T* y = static_cast<T*>(a.g.y) + (m0 + m) * a.g.ldy + o;
    const T* bias = static_cast<const T*>(a.g.bias);
    const float sums[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (o + k < a.g.l.O) y[k] = W4Type<F16>::round(bias ? sums[k] + static_cast<float>(bias[o + k]) : sums[k]);
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
// Tensor map of the rows of x, fetched in boxes of n rows x 64 columns.
bool encode_x(CUtensorMap* tm, const W4Gemm& g, int n, bool f16)
{
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const long long pitch = g.M == 1 ? (g.l.K + 7) & ~7 : g.ldx;       // one row: any pitch that the map takes
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(g.l.K), static_cast<cuuint64_t>(g.M)}, strides[1] = {static_cast<cuuint64_t>(pitch) * 2};
    const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(n)}, es[2] = {1, 1};
    return fn(tm, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(g.x), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool plan(MmaTiles& a, int sms)
{
    const W4Layout& l = a.g.l;
    const int n = a.g.M <= 64 ? (a.g.M + 31) & ~31 : ((a.g.M + ceil_div(a.g.M, 128) - 1) / ceil_div(a.g.M, 128) + 31) & ~31;
    a.n = n;
    a.mts = ceil_div(a.g.M, n);
    a.ots = ceil_div(l.O, ROWS);
    const long long tiles = static_cast<long long>(a.mts) * a.ots;
    if (tiles * l.cbs > 0x7fff0000) return false;
    a.ctas = static_cast<int>(tiles * l.cbs < sms ? tiles * l.cbs : sms);
    // Cutting the last tiles saves steps of 0.6 us each and costs the parts' way through memory and the second launch, 4 us.
    const long long whole = (tiles + a.ctas - 1) / a.ctas;
    if (whole * l.cbs - tiles * l.cbs / a.ctas < 7) {
        a.waves = static_cast<int>(whole);
        a.per = 0;
    } else {
        a.waves = static_cast<int>(tiles / a.ctas > 0 ? tiles / a.ctas - 1 : 0);
        const long long steps = (tiles - static_cast<long long>(a.waves) * a.ctas) * l.cbs;
        a.per = static_cast<int>((steps + a.ctas - 1) / a.ctas);
    }
    return true;
}

template <bool F16, int NG, bool ZEROS, bool FEW>
int launch(const CUtensorMap& tx, const CUtensorMap& tw, const MmaTiles& a, cudaStream_t st)
{
    auto kernel = w4_mma_kernel<F16, NG, ZEROS, FEW>;
    const int smem = 1024 + RING * a.n * 256 + Roles<FEW>::W_STAGES * BLOCKS * a.g.l.block;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) { cudaGetLastError(); return BS_ERR_CUDA; }
    int rc = launch_dependent(kernel, dim3(a.ctas), dim3(Roles<FEW>::WARPS * 32), smem, st, tx, tw, a);
    if (rc == BS_OK && a.per > 0 && a.ctas > 1) rc = launch_dependent(w4_join_kernel<F16>, dim3(a.ctas - 1, a.n * ROWS / 1024), dim3(256), 0, st, a);
    return rc;
}
template <bool F16, bool FEW>
int launch_group(const CUtensorMap& tx, const CUtensorMap& tw, const MmaTiles& a, cudaStream_t st)
{
    const int ng = a.g.l.group == 32 ? 4 : a.g.l.group == 64 ? 2 : 1;
    if (a.g.l.zeros) return ng == 4 ? launch<F16, 4, true, FEW>(tx, tw, a, st) : ng == 2 ? launch<F16, 2, true, FEW>(tx, tw, a, st) : launch<F16, 1, true, FEW>(tx, tw, a, st);
    return ng == 4 ? launch<F16, 4, false, FEW>(tx, tw, a, st) : ng == 2 ? launch<F16, 2, false, FEW>(tx, tw, a, st) : launch<F16, 1, false, FEW>(tx, tw, a, st);
}

}  // namespace

// In elements of eight bytes, so that a block is no wider than a box may be.
bool w4_encode_blocks(CUtensorMap* tm, const void* prepared, const W4Layout& l, int matrices, int wide, int high)
{
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(l.block / 8), static_cast<cuuint64_t>(l.cbs), static_cast<cuuint64_t>(l.rbs), static_cast<cuuint64_t>(matrices)};
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(l.block), static_cast<cuuint64_t>(l.cbs) * l.block, l.bytes()};
    const cuuint32_t box[4] = {static_cast<cuuint32_t>(l.block / 8), static_cast<cuuint32_t>(wide), static_cast<cuuint32_t>(high), 1}, es[4] = {1, 1, 1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_INT64, 4, const_cast<void*>(prepared), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Up to 16 rows of x csrc/w4_gemm.cu is faster at every size.  Above, by times fitted to 81 pairs (20 to 512 rows, 256 x 512 to 8192 x 4096): there 2 us and
// 0.6 ns (groups of 32: 0.9) a block of weights and 16 rows of x; here 3.7 us, or 8.5 where tiles are cut, and for each of a CTA's steps 0.6 us with up to
// 64 rows, 0.75 with more, and up to three times that with four groups a step.
bool w4_mma_wanted(int M, const W4Layout& l, int sms)
{
    if (M <= 16) return false;
    MmaTiles a{};
    a.g.M = M;
    a.g.l = l;
    if (!plan(a, sms)) return false;
    if (ceil_div(M, 16) > 65535) return true;       // a grid has no more tiles of 16 rows
    const double step = l.group == 32 ? 1.7 : l.group == 64 ? 0.85 : a.n <= 64 ? 0.6 : 0.75;
    const double here = (a.per ? 8.5 : 3.7) + step * (static_cast<double>(a.waves) * l.cbs + a.per);
    return 2 + (l.group == 32 ? 0.9e-3 : 0.6e-3) * l.rbs * l.cbs * ceil_div(M, 16) > here;
}

size_t w4_mma_workspace(int M, const W4Layout& l, int sms)
{
    MmaTiles a{};
    a.g.M = M;
    a.g.l = l;
    return plan(a, sms) && a.per > 0 ? static_cast<size_t>(2) * a.ctas * a.n * ROWS * sizeof(float) : 0;
}

int w4_mma_launch(const W4Gemm& g, bool f16, float* part, int sms, cudaStream_t st)
{
    MmaTiles a{};
    a.g = g;
    a.part = part;
    CUtensorMap tx, tw;
    if (!plan(a, sms)) return BS_ERR_UNSUPPORTED;
    if (!encode_x(&tx, g, a.n, f16) || !w4_encode_blocks(&tw, g.w, a.g.l, 1, 1, BLOCKS)) return BS_ERR_CUDA;
    if (a.n <= 64) return f16 ? launch_group<true, true>(tx, tw, a, st) : launch_group<false, true>(tx, tw, a, st);
    return f16 ? launch_group<true, false>(tx, tw, a, st) : launch_group<false, false>(tx, tw, a, st);
}

}  // namespace bs
