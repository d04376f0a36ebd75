// Quantiser and set-up of 4-bit weights with a scale per group (layout: w4.h).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "w4.h"

namespace bs {
namespace {

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }

// Least and largest of V values and 0 (a NaN does not count): two of 16 bits at a time.
template <int V>
__device__ __forceinline__ void extremes(const float* v, float& lo, float& hi)
{
    lo = hi = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) { lo = fminf(lo, v[e]); hi = fmaxf(hi, v[e]); }
}
template <int V, typename T2>
__device__ __forceinline__ void extremes2(const T2* v, T2 zero, float& lo, float& hi)
{
    T2 l = zero, h = zero;
#pragma unroll
    for (int e = 0; e < V / 2; ++e) { l = __hmin2(l, v[e]); h = __hmax2(h, v[e]); }
    lo = fminf(to_f(l.x), to_f(l.y));
    hi = fmaxf(to_f(h.x), to_f(h.y));
}
template <int V> __device__ __forceinline__ void extremes(const __half* v, float& lo, float& hi)
{
    extremes2<V>(reinterpret_cast<const __half2*>(v), __floats2half2_rn(0.f, 0.f), lo, hi);
}
template <int V> __device__ __forceinline__ void extremes(const __nv_bfloat16* v, float& lo, float& hi)
{
    extremes2<V>(reinterpret_cast<const __nv_bfloat162*>(v), __floats2bfloat162_rn(0.f, 0.f), lo, hi);
}

template <typename S> struct Step;
template <> struct Step<__half> {
    static constexpr float MAX = 65504.f;
    static __device__ __half round(float v) { return __float2half_rn(v); }
};
template <> struct Step<__nv_bfloat16> {
    static constexpr float MAX = 3.3895313892515355e38f;
    static __device__ __nv_bfloat16 round(float v) { return __float2bfloat16_rn(v); }
};

// clip(round_half_even(w / s)) of the Section IV quantiser for the values of one group, of the exact quotient; a NaN gets the lowest code (fmaxf returns the
// other operand).  The quotient is w times the reciprocal, corrected once by its residual: exact where it is a tie, because a tie is a float, and
// for weights of 16 bits on the right side everywhere else, because a quotient of theirs that is no tie is 2^-17 of it away.  For float32
// weights the exact residual tells the side of what rounds to a tie.  Groups with infinite weights or a scale whose reciprocal a float does not
// hold well take the division, which made the quantiser four times as slow as its bytes.
template <bool F32>
struct GroupCodes {
    float s, r, lo, hi;
    bool divide;
    // The whole number in the last places of a float: whole() of it, or its low byte.
    static constexpr float MAGIC = 12582912.f;      // 1.5 * 2^23: a last place is one
    template <bool DIVIDE>
    __device__ __forceinline__ float place(float w) const
    {
        float q = DIVIDE ? __fdiv_rn(w, s) : w * r;
        if (!DIVIDE) q = fmaf(fmaf(-q, s, w), r, q);
        q = fminf(fmaxf(q, lo), hi);
        float m = q + MAGIC;
        if ((F32 || DIVIDE) && fabsf(q - (m - MAGIC)) == 0.5f) {
            const float left = __fmaf_rn(-q, s, w);
            if (left != 0.f) m = (q + copysignf(0.5f, left)) + MAGIC;
        }
        return m;
    }
    static __device__ __forceinline__ int whole(float m) { return static_cast<int>(__float_as_uint(m) - __float_as_uint(MAGIC)); }
};

// The scale of a group from its extremes, its zero point, and what makes codes of its values (less the zero point).
template <typename S, bool ZEROS, bool F32>
__device__ __forceinline__ GroupCodes<F32> group_step(float lo, float hi, S& scale, int& z)
{
    // clip in place of overflow: a group whose scale the type cannot hold gets the largest one (fminf also where hi - lo is infinite)
    const float span = ZEROS ? __fsub_rn(hi, lo) : fmaxf(hi, -lo);
    scale = Step<S>::round(fminf(__fdiv_rn(span, ZEROS ? 15.f : 7.f), Step<S>::MAX));
    GroupCodes<F32> g;
    g.s = to_f(scale);
    g.divide = !(g.s > 1e-30f && g.s < 1e30f && span < 1e37f);
    g.r = g.divide ? 0.f : __frcp_rn(g.s);
    g.lo = ZEROS ? 0.f : -8.f;
    g.hi = ZEROS ? 15.f : 7.f;
    z = 0;
    if (!(g.s > 0.f)) {     // every code is the zero point
        g.divide = false;
        g.lo = g.hi = 0.f;
    } else if (ZEROS) {
        z = GroupCodes<F32>::whole(g.divide ? g.template place<true>(-lo) : g.template place<false>(-lo));
        g.lo = static_cast<float>(-z);
        g.hi = static_cast<float>(15 - z);
    }
    return g;
}

// Groups of 32, 64, 128 or 256 columns: a thread keeps V columns in registers, group / V neighbouring threads share the extremes by shuffles, one pass over the
// weights.  2^log_row threads take a row, the others of the CTA the next ones.  Bound by HBM, then by the instructions of the codes: 24576 x 8192 from
// bfloat16 129 us (4.7 TB/s), with zero points 146 (4.2), from float32 169 (6.0).  WIDE: rows allow 16-byte loads, a thread's columns are neighbours, 16 of
// them where K allows, 8 otherwise (8184 columns: 215 us with zero points, of which the narrower loads and stores are the cause).  Otherwise the threads of a
// group take its columns in turn, so that a load or store of single values meets few sectors: 8191 columns 283 us with groups of 128 (neighbours: 483; a
// warp a group: 499) and 298 with groups of 32 (8 columns a thread: four threads a group; 506 with 16).
template <typename T, typename S, bool ZEROS, int V, bool WIDE>
__global__ void __launch_bounds__(256) w4_quantise_kernel(const T* w, long long ld, int O, int K, int log_group, int log_row, int8_t* codes, S* scales, int8_t* zeros)
{
    w = dependent_begin(w);
    const int group = 1 << log_group, lanes = group / V, G = (K + group - 1) >> log_group, units = G * lanes;     // threads of a row, its short last group filled up
    const int rows = blockDim.x >> log_row, t = threadIdx.x & ((1 << log_row) - 1), step = gridDim.x * rows;
    // every thread goes through the same rounds: the shuffles need whole warps
    for (int first = blockIdx.x * rows; first < O; first += step) {
        const int o = first + (threadIdx.x >> log_row);
        for (int u0 = 0; u0 < units; u0 += 1 << log_row) {
            // a thread's first column, and how far apart its columns are
            const int u = u0 + t, c0 = WIDE ? u * V : (u / lanes << log_group) + (u & (lanes - 1)), apart = WIDE ? 1 : lanes;
            const bool live = o < O && c0 < K;      // WIDE: K is a multiple of V
            uint4 raw[sizeof(T) * V / 16];
            T* v = reinterpret_cast<T*>(raw);
            const T* from = w + o * ld + c0;
            if constexpr (WIDE) {
#pragma unroll
                for (int e = 0; e < static_cast<int>(sizeof(T)) * V / 16; ++e) raw[e] = live ? __ldcs(reinterpret_cast<const uint4*>(from) + e) : make_uint4(0, 0, 0, 0);
            } else {
                const int left = live ? K - c0 : 0;
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = e * apart < left ? from[e * apart] : T(0.f);
            }
            float lo, hi;
            extremes<V>(v, lo, hi);
            for (int d = 1; d < lanes; d <<= 1) {
                lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
                hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
            }
            S scale;
            int z;
            const auto g = group_step<S, ZEROS, sizeof(T) == 4>(lo, hi, scale, z);
            if (!live) continue;
            uint32_t c[V];
            // the low byte is the code's, but for the zero point
            if (g.divide) {
#pragma unroll
                for (int e = 0; e < V; ++e) c[e] = __float_as_uint(g.template place<true>(to_f(v[e])));
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) c[e] = __float_as_uint(g.template place<false>(to_f(v[e])));
            }
            // 15 at most: the sum of a byte does not reach the next one (codes without zero points are signed and have z = 0)
            uint32_t out[V / 4];
#pragma unroll
            for (int e = 0; e < V; e += 4)
                out[e / 4] = ZEROS ? __vadd4(__byte_perm(__byte_perm(c[e], c[e + 1], 0x0040), __byte_perm(c[e + 2], c[e + 3], 0x0040), 0x5410), z * 0x01010101u)
                                   : __byte_perm(__byte_perm(c[e], c[e + 1], 0x0040), __byte_perm(c[e + 2], c[e + 3], 0x0040), 0x5410);
            int8_t* to = codes + static_cast<long long>(o) * K + c0;
            if constexpr (!WIDE) {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e * apart < K - c0) to[e * apart] = static_cast<int8_t>(out[e / 4] >> (8 * (e & 3)));
            } else if (V == 16) *reinterpret_cast<uint4*>(to) = make_uint4(out[0], out[1], out[V / 4 - 2], out[V / 4 - 1]);
            else *reinterpret_cast<uint2*>(to) = make_uint2(out[0], out[1]);
            if ((u & (lanes - 1)) == 0) {
                const long long at = static_cast<long long>(o) * G + u / lanes;
                scales[at] = scale;
                if (ZEROS) zeros[at] = static_cast<int8_t>(z);
            }
        }
    }
}

// Any other group, and any row: a warp a group, which it reads twice, from L2 or L1 the second time.  24576 x 8192 from bfloat16 with zero points, groups of
// 384: 321 us; loads and stores of single values bound it.
template <typename T, typename S, bool ZEROS>
__global__ void __launch_bounds__(256) w4_quantise_rows_kernel(const T* w, long long ld, int O, int K, int group, int8_t* codes, S* scales, int8_t* zeros)
{
    w = dependent_begin(w);
    const int lane = threadIdx.x & 31, G = (K + group - 1) / group;
    const long long total = static_cast<long long>(O) * G, step = static_cast<long long>(gridDim.x) * (blockDim.x / 32);
    for (long long i = static_cast<long long>(blockIdx.x) * (blockDim.x / 32) + threadIdx.x / 32; i < total; i += step) {
        const int o = static_cast<int>(i / G);
        const int beg = static_cast<int>(i - static_cast<long long>(o) * G) * group, end = K - beg < group ? K : beg + group;
        const T* row = w + o * ld;
        float lo = 0.f, hi = 0.f;
        for (int c = beg + lane; c < end; c += 32) {
            const float v = to_f(row[c]);
            lo = fminf(lo, v);
            hi = fmaxf(hi, v);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
        }
        S scale;
        int z;
        const auto g = group_step<S, ZEROS, sizeof(T) == 4>(lo, hi, scale, z);
        for (int c = beg + lane; c < end; c += 32) {
            const float w = to_f(row[c]);
            codes[static_cast<long long>(o) * K + c] = static_cast<int8_t>(g.whole(g.divide ? g.template place<true>(w) : g.template place<false>(w)) + z);
        }
        if (lane == 0) {
            scales[i] = scale;
            if (ZEROS) zeros[i] = static_cast<int8_t>(z);
        }
    }
}

// A thread writes the 16 bytes of (t, row): 32 codes of one row; the first of a block's 64 threads its steps too.  Set-up, once per matrix: 24576 x 8192 67 us (4.5 TB/s),
// with an odd number of columns, code by code, 146.
__global__ void __launch_bounds__(256) w4_prepare_kernel(const int8_t* codes, const uint16_t* scales, const int8_t* zeros, W4Layout l, unsigned char* out)
{
    codes = dependent_begin(codes);
    const size_t m = blockIdx.y;      // matrix
    const int G = (l.K + l.group - 1) / l.group, in_block = l.group < W4_COLS ? W4_COLS / l.group : 1;
    codes += m * l.O * l.K;
    scales += m * l.O * G;
    if (zeros) zeros += m * l.O * G;
    out += m * l.bytes();
    const long long step = static_cast<long long>(gridDim.x) * blockDim.x;
    const bool wide = (l.K & 7) == 0;
    const uint32_t offset = zeros ? 0 : 8;
    for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < static_cast<long long>(l.rbs) * l.cbs * 64; i += step) {
        // the four threads of a row are neighbours: they read 32 bytes in a row
        const long long b = i >> 6;
        const int u = static_cast<int>(i) & 63, t = u & 3, r = u >> 2;
        const int rb = static_cast<int>(b / l.cbs), cb = static_cast<int>(b - static_cast<long long>(rb) * l.cbs), o = rb * 16 + r;
        unsigned char* block = out + b * l.block;
        uint32_t word[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k0 = cb * 128 + 32 * j + 8 * t;
            uint32_t c[8];
            if (o < l.O && wide && k0 < l.K) {
                const uint2 v = *reinterpret_cast<const uint2*>(codes + static_cast<size_t>(o) * l.K + k0);
#pragma unroll
                for (int e = 0; e < 8; ++e) c[e] = ((e < 4 ? v.x : v.y) >> (8 * (e & 3))) + offset;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) c[e] = o < l.O && k0 + e < l.K ? static_cast<uint8_t>(codes[static_cast<size_t>(o) * l.K + k0 + e]) + offset : 0u;
            }
            word[j] = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) word[j] |= (c[e] & 15u) << (4 * (e / 2 + 4 * (e & 1)));
        }
        *reinterpret_cast<uint4*>(block + t * 256 + ((r & 8) | ((r & 7) ^ 2 * t)) * 16) = make_uint4(word[0], word[1], word[2], word[3]);
        if (u < 8 * in_block) {
            const int low = rb * 16 + (u & 7), high = low + 8, g = in_block > 1 ? cb * in_block + (u >> 3) : cb * 128 / l.group;
            const size_t at = static_cast<size_t>(low) * G + g, up = static_cast<size_t>(high) * G + g;
            const bool has_low = low < l.O && g < G, has_high = high < l.O && g < G;
            const uint32_t s = (has_low ? scales[at] : 0u) | (has_high ? scales[up] : 0u) << 16;
            uint32_t* steps = reinterpret_cast<uint32_t*>(block + W4_CODES);
            if (zeros) *reinterpret_cast<uint2*>(steps + 2 * u) = make_uint2(s, (has_low ? zeros[at] & 15u : 0u) | (has_high ? zeros[up] & 15u : 0u) << 16);
            else steps[u] = s;
        }
    }
}

template <typename T, typename S>
int quantise(const void* w, long long ld, int O, int K, int group, int8_t* codes, void* scales, int8_t* zeros, cudaStream_t st)
{
    const T* wt = static_cast<const T*>(w);
    S* sc = static_cast<S*>(scales);
    const int sms = device_sm_count();
    if (sms <= 0) return BS_ERR_CUDA;
    const bool wide = (K & 7) == 0 && (ld * static_cast<long long>(sizeof(T))) % 16 == 0;
    const long long most = static_cast<long long>(sms) * 32;
    if (group > 256 || (group & (group - 1)) != 0) {
        const long long want = (static_cast<long long>(O) * ceil_div(K, group) + 7) / 8;
        const dim3 grid(static_cast<unsigned>(want < most ? want : most));
        return zeros ? launch_dependent(w4_quantise_rows_kernel<T, S, true>, grid, dim3(256), 0, st, wt, ld, O, K, group, codes, sc, zeros)
                     : launch_dependent(w4_quantise_rows_kernel<T, S, false>, grid, dim3(256), 0, st, wt, ld, O, K, group, codes, sc, zeros);
    }
    const int V = (wide ? K % 16 == 0 : group >= 128) ? 16 : 8, units = ceil_div(K, group) * (group / V);
    int log_group = 5, log_row = 5;
    while (1 << log_group < group) ++log_group;
    while (1 << log_row < units && log_row < 8) ++log_row;
    const int want = ceil_div(O, 256 >> log_row);
    const dim3 grid(static_cast<unsigned>(want < most ? want : most));
    auto go = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(256), 0, st, wt, ld, O, K, log_group, log_row, codes, sc, zeros); };
    if (!wide && V == 16) return zeros ? go(w4_quantise_kernel<T, S, true, 16, false>) : go(w4_quantise_kernel<T, S, false, 16, false>);
    if (!wide) return zeros ? go(w4_quantise_kernel<T, S, true, 8, false>) : go(w4_quantise_kernel<T, S, false, 8, false>);
    if (V == 16) return zeros ? go(w4_quantise_kernel<T, S, true, 16, true>) : go(w4_quantise_kernel<T, S, false, 16, true>);
    return zeros ? go(w4_quantise_kernel<T, S, true, 8, true>) : go(w4_quantise_kernel<T, S, false, 8, true>);
}

}  // namespace
}  // namespace bs

extern "C" int bs_w4_quantise(const void* w, bs_float_t w_type, int O, int K, long long ld, int group, bs_float_t type, int8_t* codes, void* scales,
                              int8_t* zeros, void* stream)
{
    using namespace bs;
    W4Layout l;
    if (!w || !codes || !scales || O <= 0 || K <= 0 || ld < K || group <= 0) return BS_ERR_INVALID_ARG;
    if ((w_type != BS_F32 && w_type != BS_F16 && w_type != BS_BF16) || (type != BS_F16 && type != BS_BF16)) return BS_ERR_INVALID_ARG;
    if (!w4_layout(O, K, group, zeros != nullptr, l)) return BS_ERR_UNSUPPORTED;
    if (!aligned16(w) || !aligned16(codes) || !aligned16(scales) || !aligned16(zeros)) return BS_ERR_ALIGNMENT;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (type == BS_F16) {
        if (w_type == BS_F32) return quantise<float, __half>(w, ld, O, K, group, codes, scales, zeros, st);
        if (w_type == BS_F16) return quantise<__half, __half>(w, ld, O, K, group, codes, scales, zeros, st);
        return quantise<__nv_bfloat16, __half>(w, ld, O, K, group, codes, scales, zeros, st);
    }
    if (w_type == BS_F32) return quantise<float, __nv_bfloat16>(w, ld, O, K, group, codes, scales, zeros, st);
    if (w_type == BS_F16) return quantise<__half, __nv_bfloat16>(w, ld, O, K, group, codes, scales, zeros, st);
    return quantise<__nv_bfloat16, __nv_bfloat16>(w, ld, O, K, group, codes, scales, zeros, st);
}

extern "C" size_t bs_w4_bytes(int O, int K, int group, int zeros)
{
    bs::W4Layout l;
    return bs::w4_layout(O, K, group, zeros, l) ? l.bytes() : 0;
}

extern "C" int bs_w4_prepare(const int8_t* codes, const void* scales, const int8_t* zeros, int matrices, int O, int K, int group, void* out, void* stream)
{
    using namespace bs;
    W4Layout l;
    if (!codes || !scales || !out || matrices <= 0 || O <= 0 || K <= 0 || group <= 0) return BS_ERR_INVALID_ARG;
    if (matrices > 65535 || !w4_layout(O, K, group, zeros != nullptr, l)) return BS_ERR_UNSUPPORTED;
    if (!aligned16(codes) || !aligned16(scales) || !aligned16(zeros) || !aligned16(out)) return BS_ERR_ALIGNMENT;
    const int sms = device_sm_count();
    if (sms <= 0) return BS_ERR_CUDA;
    const long long want = (static_cast<long long>(l.rbs) * l.cbs * 64 + 255) / 256, most = static_cast<long long>(sms) * 16;
    return launch_dependent(w4_prepare_kernel, dim3(static_cast<unsigned>(want < most ? want : most), static_cast<unsigned>(matrices)), dim3(256), 0,
                            static_cast<cudaStream_t>(stream), codes, static_cast<const uint16_t*>(scales), zeros, l, static_cast<unsigned char*>(out));
}
