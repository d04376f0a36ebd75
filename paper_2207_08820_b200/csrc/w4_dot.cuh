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

__device__ __forceinline__ uint32_t word_of(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// A block on its way through shared memory: a warp copies ahead into a ring of stages of its own and waits for nobody else.  A lane copies the codes of its
// two rows, 16 bytes each, and of the (up to four) groups in the block one entry.
template <int NG, bool ZEROS>
struct W4Stage {
    static constexpr int ENTRY = ZEROS ? 8 : 4, BYTES = W4_BLOCK + NG * 8 * ENTRY;

    static __device__ __forceinline__ void copy(uint32_t dst, const unsigned char* matrix, const W4Layout& l, int rb, int cb, int lane)
    {
        const int r = lane >> 2, t = lane & 3;
        const unsigned char* p = matrix + (static_cast<size_t>(rb) * l.cbs + cb) * W4_BLOCK + t * 256 + r * 16;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + lane * 16), "l"(p) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 512 + lane * 16), "l"(p + 128) : "memory");
        const int g = NG > 1 ? cb * NG + t : cb * 128 / l.group;
        if (t < NG && g < l.G) {
            const unsigned char* e = matrix + l.codes_bytes() + ((static_cast<size_t>(rb) * l.G + g) * 8 + r) * ENTRY;
            asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst + W4_BLOCK + (t * 8 + r) * ENTRY), "l"(e), "n"(ENTRY) : "memory");
        }
    }
};
__device__ __forceinline__ void ring_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void ring_wait()      // all but the youngest N groups have landed, for every lane of the warp
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
    __syncwarp();
}

// What a lane needs of one block: the codes of its two rows, and the scales and zero points of the groups in it.  Groups behind the last one multiply
// zeros of x only; their entries are what the ring held before, so their scales are cleared.
template <int NG, bool ZEROS>
struct W4Tile {
    uint4 a, b;
    uint32_t scale[NG], zero[NG];

    __device__ __forceinline__ void take(uint32_t src, const W4Layout& l, int cb, int lane)
    {
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w) : "r"(src + lane * 16) : "memory");
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "r"(src + 512 + lane * 16) : "memory");
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const uint32_t at = src + W4_BLOCK + (g * 8 + (lane >> 2)) * W4Stage<NG, ZEROS>::ENTRY;
            if (ZEROS) {
                asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(scale[g]), "=r"(zero[g]) : "r"(at) : "memory");
                zero[g] &= 0x000f000fu;     // what is left of an earlier block in an entry that has none stays a code
            } else {
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(scale[g]) : "r"(at) : "memory");
            }
            if (NG > 1 && g > 0 && cb * NG + g >= l.G) scale[g] = 0;
        }
    }
};

// tot[n] += the block times x[n], n tiles of eight rows of x; x[n][j]: the lane's eight columns of word j.  x is of the type that X16 says, the scales
// of S16's.
template <bool X16, bool S16, int NG, bool ZEROS, int NT>
__device__ __forceinline__ void w4_block(const W4Tile<NG, ZEROS>& w, const uint4 (&x)[NT][4], float (&tot)[NT][4])
{
    typedef W4Type<X16> Ty;
    float acc[NT][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int g = j * NG / 4;
        uint32_t z0 = Ty::BASE + 0x00080008u, z1 = z0;
        if (ZEROS) {
            z0 = Ty::BASE + __byte_perm(w.zero[g], 0, 0x1010);
            z1 = Ty::BASE + __byte_perm(w.zero[g], 0, 0x3232);
        }
        if (j % (4 / NG) == 0) {
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
        }
        const uint32_t a = word_of(w.a, j), b = word_of(w.b, j);
        const uint32_t a0 = Ty::centre(a, z0), a1 = Ty::centre(a >> 4, z0), a2 = Ty::centre(a >> 8, z0), a3 = Ty::centre(a >> 12, z0);
        const uint32_t b0 = Ty::centre(b, z1), b1 = Ty::centre(b >> 4, z1), b2 = Ty::centre(b >> 8, z1), b3 = Ty::centre(b >> 12, z1);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            Ty::mma(acc[n], a0, b0, a1, b1, x[n][j].x, x[n][j].y);
            Ty::mma(acc[n], a2, b2, a3, b3, x[n][j].z, x[n][j].w);
        }
        if ((j + 1) % (4 / NG) == 0) {      // the group's sums are scaled in 32 bits
            const float s0 = W4Type<S16>::lo(w.scale[g]), s1 = W4Type<S16>::hi(w.scale[g]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                tot[n][0] = fmaf(acc[n][0], s0, tot[n][0]);
                tot[n][1] = fmaf(acc[n][1], s0, tot[n][1]);
                tot[n][2] = fmaf(acc[n][2], s1, tot[n][2]);
                tot[n][3] = fmaf(acc[n][3], s1, tot[n][3]);
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

}  // namespace bs
