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

template <typename S> struct Step;
template <> struct Step<__half> {
    static constexpr float MAX = 65504.f;
    static __device__ __half round(float v) { return __float2half_rn(v); }
};
template <> struct Step<__nv_bfloat16> {
    static constexpr float MAX = 3.3895313892515355e38f;
    static __device__ __nv_bfloat16 round(float v) { return __float2bfloat16_rn(v); }
};

// Nearest whole number of the exact quotient w / s (s > 0), ties to even.  The rounded quotient can sit on a tie that the exact one misses: the
// residual, exact in one fused multiply-add where the quotient is small enough to matter, tells the side.
__device__ __forceinline__ float nearest_quotient(float w, float s)
{
    const float q = __fdiv_rn(w, s), n = rintf(q);
    if (fabsf(q) < 64.f && fabsf(q - truncf(q)) == 0.5f) {
        const float left = __fmaf_rn(-q, s, w);
        if (left > 0.f) return ceilf(q);
        if (left < 0.f) return floorf(q);
    }
    return n;
}

// The scale of a group from its extremes, and its zero point.
template <typename S, bool ZEROS>
__device__ __forceinline__ void group_step(float lo, float hi, S& scale, float& s, float& z)
{
    // clip in place of overflow: a group whose scale the type cannot hold gets the largest one (fminf also where hi - lo is infinite)
    const float wide = ZEROS ? __fdiv_rn(__fsub_rn(hi, lo), 15.f) : __fdiv_rn(fmaxf(hi, -lo), 7.f);
    scale = Step<S>::round(fminf(wide, Step<S>::MAX));
    s = to_f(scale);
    z = ZEROS && s > 0.f ? fminf(fmaxf(nearest_quotient(-lo, s), 0.f), 15.f) : 0.f;
}

// round_half_even(clip) of the Section IV quantiser; a NaN gets the lowest code (fmaxf returns the other operand).
template <bool ZEROS>
__device__ __forceinline__ int group_code(float w, float s, float z)
{
    if (!(s > 0.f)) return static_cast<int>(z);
    const float q = nearest_quotient(w, s) + z;
    return ZEROS ? static_cast<int>(fminf(fmaxf(q, 0.f), 15.f)) : static_cast<int>(fminf(fmaxf(q, -8.f), 7.f));
}

// Groups of 32, 64, 128 or 256 columns of rows that allow wide loads: a thread keeps eight columns in registers, group / 8 neighbouring threads
// share the extremes by shuffles, one pass over the weights.  Bound by HBM.
template <typename T, typename S, bool ZEROS>
__global__ void __launch_bounds__(256) w4_quantise_kernel(const T* w, long long ld, int O, int K, int group, int8_t* codes, S* scales, int8_t* zeros)
{
    w = dependent_begin(w);
    constexpr int V = 8;
    const int lanes = group / V, per_row = (K + group - 1) / group * lanes;      // threads of a row, its short last group filled up
    const long long total = static_cast<long long>(O) * per_row;
    const long long first = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x, step = static_cast<long long>(gridDim.x) * blockDim.x;
    const long long rounds = (total + step - 1) / step;                     // the same for every thread: the shuffles need whole warps
    for (long long k = 0; k < rounds; ++k) {
        const long long i = first + k * step;
        const int o = total >> 31 ? static_cast<int>(i / per_row) : static_cast<int>(static_cast<unsigned>(i) / static_cast<unsigned>(per_row));
        const int u = static_cast<int>(i - static_cast<long long>(o) * per_row), c0 = u * V;
        const bool live = i < total && c0 < K;      // K is a multiple of eight here
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 0.f;
        if (live) {
            const T* src = w + o * ld + c0;
            uint4 raw[sizeof(T) * V / 16];
#pragma unroll
            for (int e = 0; e < static_cast<int>(sizeof(T)) * V / 16; ++e) raw[e] = __ldcs(reinterpret_cast<const uint4*>(src) + e);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = to_f(reinterpret_cast<const T*>(raw)[e]);
        }
        float lo = 0.f, hi = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) { lo = fminf(lo, v[e]); hi = fmaxf(hi, v[e]); }
        for (int d = 1; d < lanes; d <<= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
        }
        S scale;
        float s, z;
        group_step<S, ZEROS>(lo, hi, scale, s, z);
        if (!live) continue;
        uint32_t out[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < V; ++e) out[e >> 2] |= (static_cast<uint32_t>(group_code<ZEROS>(v[e], s, z)) & 255u) << (8 * (e & 3));
        *reinterpret_cast<uint2*>(codes + static_cast<long long>(o) * K + c0) = make_uint2(out[0], out[1]);
        if (u % lanes == 0) {
            const long long at = static_cast<long long>(o) * (per_row / lanes) + u / lanes;
            scales[at] = scale;
            if (ZEROS) zeros[at] = static_cast<int8_t>(z);
        }
    }
}

// Any group and any row: a warp a group, which it reads twice.
template <typename T, typename S, bool ZEROS>
__global__ void __launch_bounds__(256) w4_quantise_rows_kernel(const T* w, long long ld, int O, int K, int group, int8_t* codes, S* scales, int8_t* zeros)
{
    w = dependent_begin(w);
    const int lane = threadIdx.x & 31, G = (K + group - 1) / group;
    const long long total = static_cast<long long>(O) * G, step = static_cast<long long>(gridDim.x) * (blockDim.x / 32);
    for (long long i = static_cast<long long>(blockIdx.x) * (blockDim.x / 32) + threadIdx.x / 32; i < total; i += step) {
        const int o = static_cast<int>(i / G), g = static_cast<int>(i - static_cast<long long>(o) * G);
        const int beg = g * group, end = K - beg < group ? K : beg + group;
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
        float s, z;
        group_step<S, ZEROS>(lo, hi, scale, s, z);
        for (int c = beg + lane; c < end; c += 32) codes[static_cast<long long>(o) * K + c] = static_cast<int8_t>(group_code<ZEROS>(to_f(row[c]), s, z));
        if (lane == 0) {
            scales[i] = scale;
            if (ZEROS) zeros[i] = static_cast<int8_t>(z);
        }
    }
}

// A thread writes the 16 bytes of (t, row): 32 codes of one row; the first of a block's 64 threads its steps too.  Set-up, once per matrix.
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
    const bool wide = group <= 256 && (group & (group - 1)) == 0 && (K & 7) == 0 && (ld * static_cast<long long>(sizeof(T))) % 16 == 0;
    const long long threads = static_cast<long long>(O) * ceil_div(K, group) * (wide ? group / 8 : 32);
    const long long want = (threads + 255) / 256, most = static_cast<long long>(sms) * 32;
    const dim3 grid(static_cast<unsigned>(want < most ? want : most));
    if (wide) return zeros ? launch_dependent(w4_quantise_kernel<T, S, true>, grid, dim3(256), 0, st, wt, ld, O, K, group, codes, sc, zeros)
                           : launch_dependent(w4_quantise_kernel<T, S, false>, grid, dim3(256), 0, st, wt, ld, O, K, group, codes, sc, zeros);
    return zeros ? launch_dependent(w4_quantise_rows_kernel<T, S, true>, grid, dim3(256), 0, st, wt, ld, O, K, group, codes, sc, zeros)
                 : launch_dependent(w4_quantise_rows_kernel<T, S, false>, grid, dim3(256), 0, st, wt, ld, O, K, group, codes, sc, zeros);
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
