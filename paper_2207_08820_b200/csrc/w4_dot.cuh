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

// Where a lane finds the blocks of 16 rows.  Weights go straight to registers, a few blocks ahead of their use, and past L1, which x needs.
template <int NG, bool ZEROS>
struct W4Rows {
    static constexpr int ENTRY = ZEROS ? 8 : 4;
    const unsigned char *codes, *steps;

    __device__ __forceinline__ W4Rows() {}
    __device__ __forceinline__ W4Rows(const unsigned char* matrix, const W4Layout& l, int rb, int lane)
    {
        codes = matrix + static_cast<size_t>(rb) * l.cbs * W4_BLOCK + (lane & 3) * 256 + (lane >> 2) * 16;
        steps = matrix + l.codes_bytes() + (static_cast<size_t>(rb) * l.G * 8 + (lane >> 2)) * ENTRY;
    }
    __device__ __forceinline__ void load(W4Tile<NG, ZEROS>& w, const W4Layout& l, int cb) const
    {
        const unsigned char* p = codes + static_cast<unsigned>(cb) * W4_BLOCK;
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w.a.x), "=r"(w.a.y), "=r"(w.a.z), "=r"(w.a.w) : "l"(p));
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w.b.x), "=r"(w.b.y), "=r"(w.b.z), "=r"(w.b.w) : "l"(p + 128));
        const int g0 = NG > 1 ? cb * NG : l.per_group == 0 ? cb : static_cast<int>(__umulhi(cb, l.per_group));
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            // groups behind the last one multiply zeros of x: their scale is one too
            const bool live = NG == 1 || g == 0 || g0 + g < l.G;
            const unsigned char* e = steps + static_cast<unsigned>(live ? g0 + g : g0) * (8 * ENTRY);
            if (ZEROS) asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w.scale[g]), "=r"(w.zero[g]) : "l"(e));
            else asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(w.scale[g]) : "l"(e));
            if (!live) w.scale[g] = 0;
        }
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
