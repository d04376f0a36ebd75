// Products of blocks of 4-bit weights with 16-bit activations in registers, by mma.sync: what the kernels for few rows of x share.
//
// A warp multiplies 16 rows by 128 columns (one block, 1 KB) with eight rows of x at a time.  Lane 4 g + t holds the codes of rows g and g + 8 in columns
// 32 j + 8 t + (0..7), word j of 16 bytes each; the reduction may run in any order, so these eight columns take the places of a fragment's columns
// 2 t, 2 t + 1, 2 t + 8 and 2 t + 9 of two steps of 16, and x is fetched in the same order: 16 bytes of row g for each word j.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "w4.h"

namespace bs {

// The eight codes of a word as four pairs of numbers (code - zero point) / PART, exact.  A code in a mantissa's lowest four bits under a fixed exponent is 128 +
// code (bf16) or 1024 + code (fp16); four bits up it is 1024 + 16 code in fp16, and in bf16, whose mantissa ends there, a number below or just above the
// smallest normal one, where numbers are evenly spaced: code 2^-129.  One fused operation takes either to (code - zero point) / PART, a whole
// number of at most four bits and a sign in quarters (bf16) or ones.  So a word costs four masks, one shift and four of these; logic and shifts go
// through a pipe of half rate, which bounds these kernels.
template <bool F16> struct W4Type;
template <> struct W4Type<false> {
    typedef __nv_bfloat16 T;
    static constexpr float PART = 4.f;
    // z: the zero point in both halves
    static __device__ __forceinline__ void pairs(uint32_t w, uint32_t z, uint32_t (&v)[4])
    {
        const uint32_t h = w >> 8;
        const uint32_t u[4] = {(w & 0x000f000fu) | 0x43004300u, w & 0x00f000f0u, (h & 0x000f000fu) | 0x43004300u, h & 0x00f000f0u};
        const uint32_t quarter = 0x3e803e80u, most = 0x7f007f00u, t32 = 0x42004200u, high = 0xc200c200u + z;      // most: 2^127; high: -(128 + zero) / 4
        const __nv_bfloat162 low = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&high), *reinterpret_cast<const __nv_bfloat162*>(&t32));     // -zero / 4
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = *reinterpret_cast<const __nv_bfloat162*>(&u[i]);
            const __nv_bfloat162 d = i & 1 ? __hfma2(b, *reinterpret_cast<const __nv_bfloat162*>(&most), low)
                                           : __hfma2(b, *reinterpret_cast<const __nv_bfloat162*>(&quarter), *reinterpret_cast<const __nv_bfloat162*>(&high));
            v[i] = *reinterpret_cast<const uint32_t*>(&d);
        }
    }
    static __device__ __forceinline__ float lo(uint32_t v) { return __uint_as_float(v << 16); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
    static __device__ __forceinline__ T round(float v) { return __float2bfloat16_rn(v); }
    static __device__ __forceinline__ uint32_t round2(float lo, float hi)
    {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
    {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};
template <> struct W4Type<true> {
    typedef __half T;
    static constexpr float PART = 1.f;
    static constexpr uint32_t BASE = 0x64006400u;
    static __device__ __forceinline__ void pairs(uint32_t w, uint32_t z, uint32_t (&v)[4])
    {
        const uint32_t u[4] = {(w & 0x000f000fu) | BASE, (w & 0x00f000f0u) | BASE, (w >> 8 & 0x000f000fu) | BASE, (w >> 8 & 0x00f000f0u) | BASE};
        const uint32_t zero = BASE + z, low = 0xd400d400u + 16 * z, sixteenth = 0x2c002c00u;        // low: -(64 + zero)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = *reinterpret_cast<const __half2*>(&u[i]);
            const __half2 d = i & 1 ? __hfma2(h, *reinterpret_cast<const __half2*>(&sixteenth), *reinterpret_cast<const __half2*>(&low))
                                    : __hsub2(h, *reinterpret_cast<const __half2*>(&zero));
            v[i] = *reinterpret_cast<const uint32_t*>(&d);
        }
    }
    static __device__ __forceinline__ float lo(uint32_t v) { return __low2float(*reinterpret_cast<const __half2*>(&v)); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __high2float(*reinterpret_cast<const __half2*>(&v)); }
    static __device__ __forceinline__ T round(float v) { return __float2half_rn(v); }
    static __device__ __forceinline__ uint32_t round2(float lo, float hi)
    {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
    {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};

// Read-only loads may move above the wait for the kernel before unless their address comes from behind it: pointers go through this there.
template <typename T>
__device__ __forceinline__ const T* behind_wait(const void* p)
{
    asm volatile("" : "+l"(p) : : "memory");
    return static_cast<const T*>(p);
}

__device__ __forceinline__ uint32_t word_of(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// What a lane needs of one block: the codes of its two rows, and the scales and zero points of the (up to four) groups in it.
template <int NG, bool ZEROS>
struct W4Tile {
    uint4 a, b;
    uint32_t scale[NG], zero[NG];
};

// Blocks on their way through the shared memory of a CTA: a stage holds, for each of NB matrices, WARPS blocks, one a warp.  The `split` warps of a team share
// the reduction of 16 rows, WARPS / split teams take neighbouring rows.  One thread fills stages ahead of the warps that read them, with one tensor copy of
// all teams' blocks: copies of 8 KB reach 5.7 TB/s, where a hundred of 1 KB in flight on every SM reach 3 (measured, 104 MB), and a copy takes its
// thread 130 cycles to start.  (Loads into registers a few blocks ahead wait for one another: the waits of a warp are counted in six places only.)
template <int NG, bool ZEROS, int NB, int WARPS, int STAGES>
struct W4TeamRing {
    static constexpr int ENTRY = ZEROS ? 8 : 4, BLOCK = W4_CODES + NG * 8 * ENTRY, BYTES = STAGES * NB * WARPS * BLOCK;
    static constexpr int STAGE = NB * WARPS * BLOCK;
    uint32_t base, bar;         // stages; barriers [full, empty][STAGES], whose memory holds nothing else: only an invalidated one may be written over
    uint32_t at, step;          // of the current stage: the warp's first block, as its lane reads codes and steps
    int stage;
    unsigned phase, limit;      // parity of the round; polls of a wait, 1 after one has run out

    // bars: [2 STAGES].  All threads of the CTA.
    __device__ __forceinline__ W4TeamRing(unsigned char* smem, uint64_t* bars, int warp, int lane) : stage(0), phase(0), limit(1u << 20)
    {
        base = static_cast<uint32_t>(__cvta_generic_to_shared(smem));
        bar = static_cast<uint32_t>(__cvta_generic_to_shared(bars));
        at = base + warp * BLOCK + (lane & 3) * 256 + ((lane >> 2) ^ 2 * (lane & 3)) * 16;
        step = base + warp * BLOCK + W4_CODES + (lane >> 2) * ENTRY;
        if (threadIdx.x == 0) {
            for (int s = 0; s < STAGES; ++s) {
                asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar + 8 * s) : "memory");
                asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar + 8 * (STAGES + s)), "r"(WARPS) : "memory");
            }
            asm volatile("fence.mbarrier_init.release.cluster;\n\tfence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncthreads();
    }
    __device__ __forceinline__ void next()
    {
        ++stage;
        bar += 8;
        at += STAGE;
        step += STAGE;
        if (stage == STAGES) {
            stage = 0;
            bar -= 8 * STAGES;
            at -= STAGES * STAGE;
            step -= STAGES * STAGE;
            phase ^= 1;
        }
    }
    // Bounded wait; one that runs out sets the status word, later ones then poll once.
    static __device__ __forceinline__ bool poll(uint32_t on, unsigned parity)
    {
        unsigned there;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(there) : "r"(on), "r"(parity) : "memory");
        return there;
    }
    __device__ __forceinline__ void wait(uint32_t on, unsigned parity, int* status)
    {
        if (poll(on, parity)) return;       // mostly there: nothing is counted
        for (unsigned left = limit; left > 0; --left)
            if (poll(on, parity)) return;
        if (limit > 1) atomicOr(status, STATUS_TIMEOUT);
        limit = 1;
    }
    // The producer's thread: once the stage is free, the blocks from (c, rb) on of matrix e of each of the NB tensor maps.
    __device__ __forceinline__ void fill(const CUtensorMap* const (&maps)[NB], const int (&rb)[NB], int c, int e, int* status)
    {
        wait(bar + 8 * STAGES, phase ^ 1, status);
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "n"(STAGE) : "memory");
#pragma unroll
        for (int m = 0; m < NB; ++m)
            asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                         ::"r"(base + stage * STAGE + m * WARPS * BLOCK), "l"(reinterpret_cast<uint64_t>(maps[m])), "r"(bar), "r"(0), "r"(c), "r"(rb[m]), "r"(e) : "memory");
        next();
    }
    // The same blocks on their way to L2, which may begin before the kernel in front has ended: whatever it writes there later, L2 holds.
    static __device__ __forceinline__ void hint(const CUtensorMap* map, int rb, int c, int e)
    {
        asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(c), "r"(rb), "r"(e) : "memory");
    }
    // Behind the last one: no copy outlives the CTA, whatever the warps waited for.
    __device__ __forceinline__ void drain(int filled, int* status)
    {
        limit = 1u << 20;
        for (int i = 0; i < STAGES && i < filled; ++i) {
            if (stage == 0) {
                stage = STAGES;
                bar += 8 * STAGES;
                phase ^= 1;
            }
            --stage;
            bar -= 8;
            wait(bar, phase, status);
        }
    }
    // The warps: the stage has landed; a warp's blocks of it; the warp has what it needs.
    __device__ __forceinline__ void landed(int* status) { wait(bar, phase, status); }
    __device__ __forceinline__ void take(W4Tile<NG, ZEROS> (&w)[NB]) const
    {
#pragma unroll
        for (int m = 0; m < NB; ++m) {
            const uint32_t c = at + m * WARPS * BLOCK;
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[m].a.x), "=r"(w[m].a.y), "=r"(w[m].a.z), "=r"(w[m].a.w) : "r"(c) : "memory");
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[m].b.x), "=r"(w[m].b.y), "=r"(w[m].b.z), "=r"(w[m].b.w) : "r"(c + 128) : "memory");
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const uint32_t e = step + m * WARPS * BLOCK + g * 8 * ENTRY;
                if (ZEROS) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[m].scale[g]), "=r"(w[m].zero[g]) : "r"(e) : "memory");
                else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[m].scale[g]) : "r"(e) : "memory");
            }
        }
    }
    __device__ __forceinline__ void release(int lane) const
    {
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar + 8 * STAGES) : "memory");
    }
};

// tot[r][n] += 1 / PART (of X16's type) of RT blocks of different rows times n tiles of eight rows of x: x(n, j, term) are the lane's eight columns of word j,
// of which there are TERMS to be added up.  x is of the type that X16 says, the scales of S16's.  What adds the warps' parts up multiplies by PART.
template <bool X16, bool S16, int TERMS, int RT, int NT, int NG, bool ZEROS, typename X>
__device__ __forceinline__ void w4_blocks(const W4Tile<NG, ZEROS> (&w)[RT], const X& x, float (&tot)[RT][NT][4])
{
    typedef W4Type<X16> Ty;
    float acc[RT][NT][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int g = j * NG / 4;
        uint4 v[TERMS][NT];
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n) v[t][n] = x(n, j, t);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            uint32_t z0 = 0x00080008u, z1 = z0;
            if (ZEROS) {
                z0 = __byte_perm(w[r].zero[g], 0, 0x1010);
                z1 = __byte_perm(w[r].zero[g], 0, 0x3232);
            }
            if (j % (4 / NG) == 0) {
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[r][n][0] = acc[r][n][1] = acc[r][n][2] = acc[r][n][3] = 0.f;
            }
            uint32_t a[4], b[4];
            Ty::pairs(word_of(w[r].a, j), z0, a);
            Ty::pairs(word_of(w[r].b, j), z1, b);
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    Ty::mma(acc[r][n], a[0], b[0], a[1], b[1], v[t][n].x, v[t][n].y);
                    Ty::mma(acc[r][n], a[2], b[2], a[3], b[3], v[t][n].z, v[t][n].w);
                }
            if ((j + 1) % (4 / NG) == 0) {      // the group's sums are scaled in 32 bits
                const float s0 = W4Type<S16>::lo(w[r].scale[g]), s1 = W4Type<S16>::hi(w[r].scale[g]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    tot[r][n][0] = fmaf(acc[r][n][0], s0, tot[r][n][0]);
                    tot[r][n][1] = fmaf(acc[r][n][1], s0, tot[r][n][1]);
                    tot[r][n][2] = fmaf(acc[r][n][2], s1, tot[r][n][2]);
                    tot[r][n][3] = fmaf(acc[r][n][3], s1, tot[r][n][3]);
                }
            }
        }
    }
}

// Eight columns of a row of x from k0 on, zeros behind K; a 16-byte load where the whole of them is there.
template <typename T>
__device__ __forceinline__ uint4 load_x(const T* row, int k0, int K)
{
    if (k0 + 8 <= K) return __ldg(reinterpret_cast<const uint4*>(row + k0));
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = k0 + i < K ? __ldg(reinterpret_cast<const uint16_t*>(row) + k0 + i) : 0;
    return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
}

// The lane's columns of block cb of a row, whose address includes the lane's first column: v[j] for word j.  `full`: the whole block lies before K.
template <typename T>
__device__ __forceinline__ void load_block_x(uint4 (&v)[4], const T* row, int cb, int K, bool full, int lane)
{
    row += cb * W4_COLS;
    if (full) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __ldg(reinterpret_cast<const uint4*>(row + 32 * j));
    } else {
        const int left = K - cb * W4_COLS - 8 * (lane & 3);     // columns from the lane's first one on; none at all behind the last block
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = load_x(row, 32 * j, left);
    }
}

}  // namespace bs
