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

// The pair of codes in bits 0-3 and 16-19 of `w` as two numbers less the zero point, exact: 128 + code (bf16) or 1024 + code (fp16) is the
// code under a fixed exponent, and the difference to 128 + zero or 1024 + zero is a whole number of at most four bits and a sign.
template <bool F16> struct W4Type;
template <> struct W4Type<false> {
    typedef __nv_bfloat16 T;
    static constexpr uint32_t BASE = 0x43004300u;
    static __device__ __forceinline__ uint32_t centre(uint32_t w, uint32_t zero)
    {
        const uint32_t v = (w & 0x000f000fu) | BASE;
        const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&zero));
        return *reinterpret_cast<const uint32_t*>(&d);
    }
    static __device__ __forceinline__ float lo(uint32_t v) { return __uint_as_float(v << 16); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
    static __device__ __forceinline__ T round(float v) { return __float2bfloat16_rn(v); }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
    {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};
template <> struct W4Type<true> {
    typedef __half T;
    static constexpr uint32_t BASE = 0x64006400u;
    static __device__ __forceinline__ uint32_t centre(uint32_t w, uint32_t zero)
    {
        const uint32_t v = (w & 0x000f000fu) | BASE;
        const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&zero));
        return *reinterpret_cast<const uint32_t*>(&d);
    }
    static __device__ __forceinline__ float lo(uint32_t v) { return __low2float(*reinterpret_cast<const __half2*>(&v)); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __high2float(*reinterpret_cast<const __half2*>(&v)); }
    static __device__ __forceinline__ T round(float v) { return __float2half_rn(v); }
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

// Blocks on their way through shared memory: a warp copies ahead into a ring of STAGES of its own, RT blocks a stage, one bulk copy each, and waits for
// nobody else.  (Loads into registers a few blocks ahead wait for one another: the waits of a warp are counted in six places only.)
template <int NG, bool ZEROS, int RT, int STAGES>
struct W4Ring {
    static constexpr int ENTRY = ZEROS ? 8 : 4, BLOCK = W4_CODES + NG * 8 * ENTRY, BYTES = STAGES * RT * BLOCK;
    uint32_t base, bars;        // the barriers' memory holds nothing else: only an invalidated one may be written over
    int in, out;                // stages that are filled and read next
    unsigned phase, limit;      // parity of the round of `out`; polls of a wait, 1 after one has run out

    __device__ __forceinline__ W4Ring(unsigned char* smem, uint64_t (&bar)[STAGES], int warp, int lane) : in(0), out(0), phase(0), limit(1u << 20)
    {
        base = static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + warp * BYTES;
        bars = static_cast<uint32_t>(__cvta_generic_to_shared(bar));
        if (lane == 0) {
#pragma unroll
            for (int s = 0; s < STAGES; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + 8 * s) : "memory");
            asm volatile("fence.mbarrier_init.release.cluster;\n\tfence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
    }
    // Fills the next stage with the blocks at p; every lane has read what it held.
    __device__ __forceinline__ void put(const unsigned char* const (&p)[RT], int lane)
    {
        if (lane == 0) {
            const uint32_t bar = bars + 8 * in;
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "n"(RT * BLOCK) : "memory");
#pragma unroll
            for (int r = 0; r < RT; ++r)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                             ::"r"(base + (in * RT + r) * BLOCK), "l"(p[r]), "n"(BLOCK), "r"(bar) : "memory");
        }
        in = in + 1 == STAGES ? 0 : in + 1;
    }
    // The blocks of the next stage that was filled.  A wait that runs out sets the status word; later ones then poll once.
    __device__ __forceinline__ void get(W4Tile<NG, ZEROS> (&w)[RT], int lane, int* status)
    {
        const uint32_t bar = bars + 8 * out;
        unsigned ok = 0;
        for (unsigned it = 0; it < limit && !ok; ++it)
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(phase) : "memory");
        if (!ok) {
            if (limit > 1) atomicOr(status, STATUS_TIMEOUT);
            limit = 1;
        }
        __syncwarp();
        const int r8 = lane >> 2, t = lane & 3;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const uint32_t block = base + (out * RT + r) * BLOCK, at = block + t * 256 + (r8 ^ 2 * t) * 16;
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[r].a.x), "=r"(w[r].a.y), "=r"(w[r].a.z), "=r"(w[r].a.w) : "r"(at) : "memory");
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[r].b.x), "=r"(w[r].b.y), "=r"(w[r].b.z), "=r"(w[r].b.w) : "r"(at + 128) : "memory");
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const uint32_t step = block + W4_CODES + (g * 8 + r8) * ENTRY;
                if (ZEROS) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[r].scale[g]), "=r"(w[r].zero[g]) : "r"(step) : "memory");
                else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[r].scale[g]) : "r"(step) : "memory");
            }
        }
        if (++out == STAGES) { out = 0; phase ^= 1; }
    }
};

// tot[r][n] += RT blocks of different rows times n tiles of eight rows of x: x(n, j, term) are the lane's eight columns of word j, of which there are TERMS
// to be added up.  x is of the type that X16 says, the scales of S16's.
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
            uint32_t z0 = Ty::BASE + 0x00080008u, z1 = z0;
            if (ZEROS) {
                z0 = Ty::BASE + __byte_perm(w[r].zero[g], 0, 0x1010);
                z1 = Ty::BASE + __byte_perm(w[r].zero[g], 0, 0x3232);
            }
            if (j % (4 / NG) == 0) {
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[r][n][0] = acc[r][n][1] = acc[r][n][2] = acc[r][n][3] = 0.f;
            }
            const uint32_t a = word_of(w[r].a, j), b = word_of(w[r].b, j);
            const uint32_t a0 = Ty::centre(a, z0), a1 = Ty::centre(a >> 4, z0), a2 = Ty::centre(a >> 8, z0), a3 = Ty::centre(a >> 12, z0);
            const uint32_t b0 = Ty::centre(b, z1), b1 = Ty::centre(b >> 4, z1), b2 = Ty::centre(b >> 8, z1), b3 = Ty::centre(b >> 12, z1);
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    Ty::mma(acc[r][n], a0, b0, a1, b1, v[t][n].x, v[t][n].y);
                    Ty::mma(acc[r][n], a2, b2, a3, b3, v[t][n].z, v[t][n].w);
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

// The lane's columns of block cb of a row: v[j] for word j.  `full`: the whole block lies before K.
template <typename T>
__device__ __forceinline__ void load_block_x(uint4 (&v)[4], const T* row, int cb, int K, bool full, int lane)
{
    const int k0 = cb * W4_COLS + 8 * (lane & 3);
    if (full) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __ldg(reinterpret_cast<const uint4*>(row + k0 + 32 * j));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = load_x(row, k0 + 32 * j, K);
    }
}

}  // namespace bs
