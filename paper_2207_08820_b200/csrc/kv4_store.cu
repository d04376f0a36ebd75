// Keys and values of new tokens into pages of 4-bit codes, and the values that codes stand for out of them.
//
// A vector of `group` channels is c s + m: m its least value, s a fifteenth of its span.  Half a warp takes one token of one head, eight channels a
// lane; a CTA takes neighbouring tokens of one head, whose entries lie side by side.  A code is the product with the reciprocal, rounded; what it leaves of the
// difference, x - m - c s, is exact in binary32 and shows whether the quotient was rounded the right way: it is compared with s / 2.  On that border
// what the subtraction x - m lost decides, then half-even.
//
// The values' rows hold nibble i of eight channels 8 i + g in part g (kv4.h): eight lanes with a word of nibbles each exchange them in three steps.
#include "kv4.h"
#include "mma_kernel.cuh"
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int THREADS = 256, ROWS = THREADS / 16;

struct Rows {                   // [T][H] vectors of D values, as far apart as the caller has them
    const void* k;
    const void* v;
    long long k_token, k_head, v_token, v_head;
};
struct Store {
    Kv4 l;
    Kv4Table t;
    const int32_t* at;
    const int32_t* starts;
    int T;
};

// Where token i of the packed ones lies, -1: nowhere.
__device__ __forceinline__ int place_of(const Store& a, int i, int& slot)
{
    const int b = kv4_sequence_of(a.starts, a.t.B, i);
    if (b >= a.t.B) return -1;
    long long entry = a.at[b];
    if (a.starts) {
        if (i < a.starts[b] || i >= a.starts[b + 1]) return -1;
        entry += static_cast<long long>(i) - a.starts[b];
    }
    if (entry < 0 || entry >= static_cast<long long>(a.t.width) * a.l.page) return -1;
    slot = static_cast<int>(entry) & (a.l.page - 1);
    return kv4_page_of(a.l, a.t, b, entry);
}

// Lane i of eight has nibbles [i][0..7], afterwards [0..7][i].
__device__ __forceinline__ uint32_t exchanged(uint32_t w)
{
    const int lane = threadIdx.x;
#pragma unroll
    for (int d = 1; d < 8; d *= 2) {
        const uint32_t low = d == 1 ? 0x0f0f0f0fu : d == 2 ? 0x00ff00ffu : 0x0000ffffu;        // nibbles whose index lacks d
        const uint32_t other = __shfl_xor_sync(0xffffffffu, w, d);
        w = lane & d ? (w & ~low) | (other >> 4 * d & low) : (w & low) | (other << 4 * d & ~low);
    }
    return w;
}

// Codes of eight values of a group that has least value m and step s, whatever they are.
__device__ __noinline__ uint32_t codes_at_borders(uint4 raw, bool f16, float m, float s)
{
    // steps near the ends of binary32 are brought to where their reciprocals and products are exact
    const float up = s < 0x1p-60f ? 0x1p64f : s > 0x1p60f ? 0x1p-64f : 1.f, t = s * up, half = 0.5f * t, inverse = __frcp_rn(t);
    uint32_t word = 0;
#pragma unroll 1
    for (int i = 7; i >= 0; --i) {
        const uint32_t w = i >= 6 ? raw.w : i >= 4 ? raw.z : i >= 2 ? raw.y : raw.x;
        const float x = f16 ? (i & 1 ? W4Type<true>::hi(w) : W4Type<true>::lo(w)) : (i & 1 ? W4Type<false>::hi(w) : W4Type<false>::lo(w)), d = x - m, e = d * up;
        float c = fminf(rintf(e * inverse), 15.f);
        const float rest = fmaf(-c, t, e), back = x - d, lost = (x - (d + back)) + (back - m);         // of the difference, exact
        const bool odd = static_cast<int>(c) & 1;
        if (rest > half || (rest == half && (lost > 0.f || (lost == 0.f && odd)))) c += 1.f;
        else if (rest < -half || (rest == -half && (lost < 0.f || (lost == 0.f && odd)))) c -= 1.f;
        word = word * 16 + static_cast<uint32_t>(fminf(fmaxf(c, 0.f), 15.f));
    }
    return s > 0.f ? word : 0u;
}

// The lesser ones of two pairs of values; a NaN stays one.
template <bool F16>
__device__ __forceinline__ uint32_t least(uint32_t a, uint32_t b)
{
    uint32_t r;
    if (F16) asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// One vector of a half warp: its codes (eight a lane, lanes from D / 8 on have none) and the group's step and offset as a word of the layout.
template <bool F16>
__device__ __forceinline__ uint32_t quantise(const uint4& raw, int group, bool live, uint32_t& step)
{
    typedef W4Type<F16> Ty;
    constexpr uint32_t SIGNS = 0x80008000u, INF = F16 ? 0x7c007c00u : 0x7f807f80u;
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    // the least value in one half, minus the largest one in the other
    const uint32_t lo = least<F16>(least<F16>(w[0], w[1]), least<F16>(w[2], w[3]));
    const uint32_t hi = least<F16>(least<F16>(w[0] ^ SIGNS, w[1] ^ SIGNS), least<F16>(w[2] ^ SIGNS, w[3] ^ SIGNS));
    uint32_t ends = live ? least<F16>(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632)) : INF;
#pragma unroll
    for (int d = 1; d < 16; d *= 2) {
        if (8 * d >= group) break;
        ends = least<F16>(ends, __shfl_xor_sync(0xffffffffu, ends, d));
    }
    const float m = Ty::lo(ends), span = -Ty::hi(ends) - m;
    if (!(span < INFINITY)) {        // a vector with an infinity or a NaN, or a span that binary32 does not hold: reads as NaN
        step = 0x7fff0000u;
        return 0;
    }
    step = Ty::round2(__fdiv_rn(span, 15.f), m);
    const float s = Ty::lo(step), inverse = __frcp_rn(s), magic = 12582912.f;       // 1.5 * 2^23: the lowest bits of a sum are the whole number
    auto both = [](float v) { return f2_pack(__float_as_uint(v), __float_as_uint(v)); };
    const u64 m2 = both(-m), s2 = both(-s), inverse2 = both(inverse), magic2 = both(magic), less2 = both(-magic);
    uint32_t code[8];
    float far = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u64 x = f2_pack(__float_as_uint(Ty::lo(w[i])), __float_as_uint(Ty::hi(w[i])));
        const u64 d = f2_add(x, m2), q = f2_fma(d, inverse2, 0), near = f2_fma(f2_fma(q, s2, d), inverse2, q), c = f2_add(near, magic2);
        uint32_t r0, r1;
        f2_split(f2_fma(f2_add(c, less2), s2, d), r0, r1);
        f2_split(c, code[2 * i], code[2 * i + 1]);
        far = fmaxf(far, fmaxf(fabsf(__uint_as_float(r0)), fabsf(__uint_as_float(r1))));
    }
    // The quotients are rounded correctly, so that ties come out half-even, where the difference is exact: no value and no offset is then below 2^-12 of the span.
    // Steps of few bits (the type's smallest) may leave quotients above 15.
    const float half = 0.5f * s;
    const uint32_t small = least<F16>(least<F16>(w[0] & ~SIGNS, w[1] & ~SIGNS), least<F16>(w[2] & ~SIGNS, w[3] & ~SIGNS));
    const bool plain = s > 0x1p-60f && s < 0x1p60f && span < 15.5f * s &&
                       (far < half || (far == half && fminf(fminf(Ty::lo(small), Ty::hi(small)), fabsf(m)) >= span * 0x1p-12f));
    if (!plain) return codes_at_borders(raw, F16, m, s);
    uint32_t word = code[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) word = word * 16 + code[i];
    return word - 0x3f400000u;          // magic's bits times 16^i, summed
}

template <bool F16>
__global__ void __launch_bounds__(THREADS) kv4_append_kernel(const __grid_constant__ Store a, const __grid_constant__ Rows r)
{
    Store b = a;
    b.t.pages = dependent_begin(a.t.pages);
    b.at = behind_wait<int32_t>(a.at);
    b.starts = behind_wait<int32_t>(a.starts);
    const uint16_t *k = behind_wait<uint16_t>(r.k), *v = behind_wait<uint16_t>(r.v);
    const int m = threadIdx.x & 15, D = a.l.D;
    const int h = blockIdx.y;
    const bool live = 8 * m < D;
    for (long long first = blockIdx.x * ROWS; first < a.T; first += gridDim.x * ROWS) {
        const int token = static_cast<int>(first) + (threadIdx.x >> 4);
        int page = -1, slot = 0;
        uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        if (token < a.T) {
            if (live) {
                x[0] = *reinterpret_cast<const uint4*>(k + token * r.k_token + h * r.k_head + 8 * m);
                x[1] = *reinterpret_cast<const uint4*>(v + token * r.v_token + h * r.v_head + 8 * m);
            }
            page = place_of(b, token, slot);
        }
        uint32_t step[2], code[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) code[j] = quantise<F16>(x[j], a.l.group, live, step[j]);
        const uint32_t part = exchanged(live ? code[1] : 0u);        // of part m & 7: nibbles 8 (m >> 3) .. + 7
        if (page < 0) continue;
        unsigned char* tile = kv4_tile_of(a.l, page, h, slot);
        const int e = slot % KV4_TILE;
        if (live) {
            *reinterpret_cast<uint32_t*>(tile + kv4_key_row(e) * (D / 2) + (m & 3) * (D / 8) + (m >> 2) * 4) = code[0];
            if (8 * m % a.l.group == 0) {
                uint32_t* steps = reinterpret_cast<uint32_t*>(tile + KV4_TILE * D) + e * a.l.G + 8 * m / a.l.group;
                steps[0] = step[0];
                steps[KV4_TILE * a.l.G] = step[1];
            }
        }
        unsigned char* to = tile + KV4_TILE * (D / 2) + e * (D / 2) + kv4_value_part(D, e, m & 7) * (D / 16) + (m >> 3) * 4;
        if (D == 96) {          // parts of six bytes
            *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(part);
            if (m < 8) *reinterpret_cast<uint16_t*>(to + 2) = static_cast<uint16_t>(part >> 16);
        } else if (m < 8 || D == 128) {
            *reinterpret_cast<uint32_t*>(to) = part;
        }
    }
}

template <bool F16>
__global__ void __launch_bounds__(THREADS) kv4_read_kernel(const __grid_constant__ Store a, uint16_t* k, uint16_t* v)
{
    typedef W4Type<F16> Ty;
    Store b = a;
    b.t.pages = dependent_begin(a.t.pages);
    b.at = behind_wait<int32_t>(a.at);
    b.starts = behind_wait<int32_t>(a.starts);
    const int m = threadIdx.x & 15, D = a.l.D;
    const int h = blockIdx.y;
    const bool live = 8 * m < D;
    for (long long first = blockIdx.x * ROWS; first < a.T; first += gridDim.x * ROWS) {
        const int token = static_cast<int>(first) + (threadIdx.x >> 4);
        int page = -1, slot = 0;
        const bool there = token < a.T;
        if (there) page = place_of(b, token, slot);
        uint32_t code[2] = {0, 0}, step[2] = {0, 0};
        if (page >= 0) {
            const unsigned char* tile = behind_wait<unsigned char>(kv4_tile_of(a.l, page, h, slot));
            const int e = slot % KV4_TILE;
            const unsigned char* from = tile + KV4_TILE * (D / 2) + e * (D / 2) + kv4_value_part(D, e, m & 7) * (D / 16) + (m >> 3) * 4;
            if (D == 96) {
                code[1] = *reinterpret_cast<const uint16_t*>(from);
                if (m < 8) code[1] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(from + 2)) << 16;
            } else if (m < 8 || D == 128) {
                code[1] = *reinterpret_cast<const uint32_t*>(from);
            }
            if (live) {
                code[0] = *reinterpret_cast<const uint32_t*>(tile + kv4_key_row(e) * (D / 2) + (m & 3) * (D / 8) + (m >> 2) * 4);
                const uint32_t* steps = reinterpret_cast<const uint32_t*>(tile + KV4_TILE * D) + e * a.l.G + 8 * m / a.l.group;
                step[0] = steps[0];
                step[1] = steps[KV4_TILE * a.l.G];
            }
        }
        code[1] = exchanged(code[1]);
        if (!there || !live) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float s = Ty::lo(step[j]), o = Ty::hi(step[j]), whole = 8388608.f;       // 2^23 under a code is 2^23 + code
            uint32_t w[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float lo = __uint_as_float((code[j] >> 8 * n & 15u) | 0x4b000000u) - whole, hi = __uint_as_float((code[j] >> (8 * n + 4) & 15u) | 0x4b000000u) - whole;
                w[n] = Ty::round2(fmaf(lo, s, o), fmaf(hi, s, o));
            }
            *reinterpret_cast<uint4*>((j == 0 ? k : v) + (static_cast<long long>(token) * a.l.H + h) * D + 8 * m) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

int check(const bs_kv4_cache* c, const int32_t* table, long long pitch, int width, int B, const int32_t* at, const int32_t* starts, int T, Store& a)
{
    if (!c || !c->data || !table || !at || width <= 0 || B <= 0 || T < 0 || pitch < width) return BS_ERR_INVALID_ARG;
    if (c->type != BS_F16 && c->type != BS_BF16) return BS_ERR_INVALID_ARG;
    if (c->pages <= 0 || c->heads <= 0 || c->D <= 0 || c->page <= 0 || c->group <= 0) return BS_ERR_INVALID_ARG;
    if (!starts && T != B) return BS_ERR_INVALID_ARG;
    if (!kv4_layout(*c, a.l)) return BS_ERR_UNSUPPORTED;
    if (!aligned16(c->data)) return BS_ERR_ALIGNMENT;
    a.t = {table, pitch, width, B};
    a.at = at;
    a.starts = starts;
    a.T = T;
    return BS_OK;
}
// Neighbouring tokens of a head a CTA, as many as fill the GPU twice.
dim3 grid_of(const Store& a)
{
    const long long blocks = ceil_div_ll(a.T, ROWS), most = ceil_div(16 * device_sm_count(), a.l.H);
    return dim3(static_cast<unsigned>(blocks < most ? blocks : most), a.l.H);
}

}  // namespace
}  // namespace bs

using namespace bs;

extern "C" size_t bs_kv4_page_bytes(int heads, int D, int page, int group)
{
    Kv4 l;
    bs_kv4_cache c{nullptr, 1, heads, D, page, group, BS_BF16};
    return kv4_layout(c, l) ? static_cast<size_t>(l.whole) : 0;
}

extern "C" int bs_kv4_append(const void* k, long long k_token, long long k_head, const void* v, long long v_token, long long v_head, int T, const bs_kv4_cache* cache,
                             const int32_t* table, long long table_pitch, int width, int B, const int32_t* at, const int32_t* starts, void* stream)
{
    Store a;
    if (!k || !v || k_token < 0 || k_head < 0 || v_token < 0 || v_head < 0) return BS_ERR_INVALID_ARG;
    const int rc = check(cache, table, table_pitch, width, B, at, starts, T, a);
    if (rc != BS_OK) return rc;
    if (!aligned16(k) || !aligned16(v) || (k_token | k_head | v_token | v_head) % 8 != 0) return BS_ERR_ALIGNMENT;
    if (T == 0) return BS_OK;
    const Rows r{k, v, k_token, k_head, v_token, v_head};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cache->type == BS_F16 ? launch_dependent(kv4_append_kernel<true>, grid_of(a), dim3(THREADS), 0, st, a, r)
                                 : launch_dependent(kv4_append_kernel<false>, grid_of(a), dim3(THREADS), 0, st, a, r);
}

extern "C" int bs_kv4_read(const bs_kv4_cache* cache, const int32_t* table, long long table_pitch, int width, int B, const int32_t* at, const int32_t* starts, int T,
                           void* k, void* v, void* stream)
{
    Store a;
    if (!k || !v) return BS_ERR_INVALID_ARG;
    const int rc = check(cache, table, table_pitch, width, B, at, starts, T, a);
    if (rc != BS_OK) return rc;
    if (!aligned16(k) || !aligned16(v)) return BS_ERR_ALIGNMENT;
    if (T == 0) return BS_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint16_t *ko = static_cast<uint16_t*>(k), *vo = static_cast<uint16_t*>(v);
    return cache->type == BS_F16 ? launch_dependent(kv4_read_kernel<true>, grid_of(a), dim3(THREADS), 0, st, a, ko, vo)
                                 : launch_dependent(kv4_read_kernel<false>, grid_of(a), dim3(THREADS), 0, st, a, ko, vo);
}
