// Keys and values of new tokens into pages of 4-bit codes, and the values that codes stand for out of them.
//
// A vector of `group` channels is c s + m: m its least value, s a fifteenth of its span.  Four lanes take one token of one head, lane t the channels 32 w + 8 t +
// (0..7), 16 bytes of each 64, so that what a group costs once is shared by many values; a CTA takes neighbouring tokens of one head, whose entries lie side
// by side.  Few tokens are spread: sixteen lanes take one, lane 4 w + t a word of 8 channels.
//
// A code is the quotient, corrected once, plus 1.5 * 2^23, which leaves the whole number, ties half-even, in the lowest bits.  That is right where the difference
// x - m is exact and, since it and the borders (c + 1/2) s then lie on a grid, no quotient is nearer to a border than its own rounding.  Words of eight values
// for which the exponents do not show that are right where x - m - c s is less than s / 2, and else left to codes_at_borders.
//
// Lane t's codes of the keys are part t of their row.  The values' rows hold nibble i of eight channels 8 i + g in part g (kv4.h): the four lanes exchange bytes,
// and each writes two parts.
//
// 131072 tokens of 8 heads, bf16, one group a head: 128 us stored (5.3 TB/s); 22950 tokens, fp16, groups of 32: 65 us stored and read back (3.8 TB/s), bound by
// the instructions of the codes, 17 a value, of which fine groups are a third.
#include "kv4.h"
#include "mma_kernel.cuh"
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int THREADS = 128;

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

// Lane t of four has bytes [t][0..3], afterwards [0..3][t].
__device__ __forceinline__ uint32_t exchanged(uint32_t w)
{
    const int t = threadIdx.x & 3;
    w = __byte_perm(w, __shfl_xor_sync(0xffffffffu, w, 1), t & 1 ? 0x3715 : 0x6240);
    return __byte_perm(w, __shfl_xor_sync(0xffffffffu, w, 2), t & 2 ? 0x3276 : 0x5410);
}
// The lower (shift 0) or upper (4) nibbles of the bytes of two words, side by side: four of a, four of b.
__device__ __forceinline__ uint32_t gathered(uint32_t a, uint32_t b, int shift)
{
    a = a >> shift & 0x0f0f0f0fu;
    b = b >> shift & 0x0f0f0f0fu;
    return __byte_perm(a | a >> 4, b | b >> 4, 0x6420);
}
// The four nibbles of a word's lower half, one a byte.
__device__ __forceinline__ uint32_t spread(uint32_t w)
{
    w = __byte_perm(w, 0, 0x4140);
    return (w | w << 4) & 0x0f0f0f0fu;
}

// Codes of eight values of a group that has least value m and step s, whatever they are; plain: the step is far from the ends of binary32 and no quotient is above
// 15.5.  Few words come here, so it is no part of their loop.
template <bool F16>
__device__ __noinline__ uint32_t codes_at_borders(uint4 raw, float m, float s, float inverse, bool plain)
{
    typedef W4Type<F16> Ty;
    const float half_step = 0.5f * s;
    uint32_t word = 0;
    if (plain) {            // all differences within half a step of their codes: no question of ties
        float far = 0.f;
#pragma unroll
        for (int i = 7; i >= 0; --i) {
            const uint32_t w = word_of(raw, i >> 1);
            const float d = (i & 1 ? Ty::hi(w) : Ty::lo(w)) - m, c = rintf(d * inverse);
            far = fmaxf(far, fabsf(fmaf(-c, s, d)));
            word = word * 16 + static_cast<uint32_t>(c);
        }
        if (far < half_step) return word;
        word = 0;
    }
    // steps near the ends of binary32 are brought to where their reciprocals and products are exact
    const float up = s < 0x1p-60f ? 0x1p64f : s > 0x1p60f ? 0x1p-64f : 1.f, t = s * up, half = 0.5f * t, over = __frcp_rn(t);
#pragma unroll 1
    for (int i = 7; i >= 0; --i) {
        const uint32_t w = i >= 6 ? raw.w : i >= 4 ? raw.z : i >= 2 ? raw.y : raw.x;
        const float x = i & 1 ? Ty::hi(w) : Ty::lo(w), d = x - m, e = d * up;
        float c = fminf(rintf(e * over), 15.f);
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

template <bool F16>
__device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b)
{
    uint32_t r;
    if (F16) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// W words of a group of channels, and the others of the vector in three more lanes (ACROSS 3), or in those and the ones 4 (7) or 4 and 8 (15) away: eight codes
// a word, and the group's step and offset as a word of the layout.
template <bool F16, int W, int ACROSS>
__device__ __forceinline__ void quantise(const uint4* raw, uint32_t* code, uint32_t& step, bool live)
{
    typedef W4Type<F16> Ty;
    constexpr uint32_t SIGNS = 0x80008000u;
    // the least value in one half, minus the largest one in the other
    uint32_t lo, hi, small[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const uint32_t l = least<F16>(least<F16>(raw[w].x, raw[w].y), least<F16>(raw[w].z, raw[w].w)), h = most<F16>(most<F16>(raw[w].x, raw[w].y), most<F16>(raw[w].z, raw[w].w));
        lo = w == 0 ? l : least<F16>(lo, l);
        hi = w == 0 ? h : most<F16>(hi, h);
        small[w] = least<F16>(least<F16>(raw[w].x & ~SIGNS, raw[w].y & ~SIGNS), least<F16>(raw[w].z & ~SIGNS, raw[w].w & ~SIGNS));
    }
    hi ^= SIGNS;
    uint32_t ends = least<F16>(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
    if (!live) ends = F16 ? 0x7c007c00u : 0x7f807f80u;          // infinities
#pragma unroll
    for (int d = 1; d <= ACROSS; d *= 2) ends = least<F16>(ends, __shfl_xor_sync(0xffffffffu, ends, d));
    const float m = Ty::lo(ends), span = -Ty::hi(ends) - m;
    if (!(span < INFINITY)) {        // a vector with an infinity or a NaN, or a span that binary32 does not hold: reads as NaN
        step = 0x7fff0000u;
#pragma unroll
        for (int w = 0; w < W; ++w) code[w] = 0;
        return;
    }
    // span / 15 rounded as a division rounds it: a quotient by the rounded reciprocal, corrected by its remainder (Markstein), right for all numbers that have an exact one
    const float fifteenth = 0x1.111112p-4f, near15 = span * fifteenth, part15 = span < 0x1p-90f ? __fdiv_rn(span, 15.f) : fmaf(fmaf(near15, -15.f, span), fifteenth, near15);
    step = Ty::round2(part15, m);
    const float s = Ty::lo(step), magic = 12582912.f;       // 1.5 * 2^23
    float inverse;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(s));
    auto both = [](float v) { return f2_pack(__float_as_uint(v), __float_as_uint(v)); };
    const u64 m2 = both(-m), s2 = both(-s), inverse2 = both(inverse), magic2 = both(magic);
    // With 2^e the power of two up to the span, a value of 2^(e - 13) (bf16: 2^(e - 16)) or more is a multiple of 2^(e - 23), as the type has 11 (8) bits; with such values
    // and such an offset differences are multiples below 2^(e + 1), which 24 bits hold, and a quotient that is not on a border is 15 * 2^-24 away from it, more than its
    // rounding of 2^-21.  (With half of that they may take 25 bits, and a difference beside a border be rounded onto it.)  Steps near the ends of binary32 have
    // no reciprocals to use, and steps of few bits (the type's smallest) may leave quotients above 15.
    const float grid = __uint_as_float(__float_as_uint(span) & 0x7f800000u) * (F16 ? 0x1p-13f : 0x1p-16f);
    const bool plain = s > 0x1p-60f && s < 0x1p60f && span < 15.5f * s;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        if (!(plain && fminf(fminf(Ty::lo(small[w]), Ty::hi(small[w])), fabsf(m)) >= grid)) {
            code[w] = codes_at_borders<F16>(raw[w], m, s, inverse, plain);
            continue;
        }
        uint32_t c8[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = word_of(raw[w], i);
            const u64 d = f2_add(f2_pack(__float_as_uint(Ty::lo(v)), __float_as_uint(Ty::hi(v))), m2), q = f2_fma(d, inverse2, 0);
            f2_split(f2_add(f2_fma(f2_fma(q, s2, d), inverse2, q), magic2), c8[2 * i], c8[2 * i + 1]);
        }
        uint32_t word = c8[7];
#pragma unroll
        for (int i = 6; i >= 0; --i) word = word * 16 + c8[i];
        code[w] = word - 0x3f400000u;          // magic's bits times 16^i, summed
    }
}

// W: words of 32 channels, D / 32; PER: of a group.  SPREAD: a word a lane, sixteen lanes a row.
template <bool F16, int W, int PER, bool SPREAD>
__global__ void __launch_bounds__(THREADS) kv4_append_kernel(const __grid_constant__ Store a, const __grid_constant__ Rows r)
{
    constexpr int D = 32 * W, G = W / PER, MINE = SPREAD ? 1 : W, ROWS = THREADS / (SPREAD ? 16 : 4);
    Store b = a;
    b.t.pages = dependent_begin(a.t.pages);
    b.at = behind_wait<int32_t>(a.at);
    b.starts = behind_wait<int32_t>(a.starts);
    const uint16_t *k = behind_wait<uint16_t>(r.k), *v = behind_wait<uint16_t>(r.v);
    const int t = threadIdx.x & 3, w0 = SPREAD ? threadIdx.x >> 2 & 3 : 0, h = blockIdx.y;
    const bool live = !SPREAD || w0 < W;
    for (long long first = static_cast<long long>(blockIdx.x) * ROWS; first < a.T; first += static_cast<long long>(gridDim.x) * ROWS) {
        const int token = static_cast<int>(first) + threadIdx.x / (THREADS / ROWS);
        int page = -1, slot = 0;
        uint4 x[2][MINE];
#pragma unroll
        for (int w = 0; w < MINE; ++w) {
            x[0][w] = x[1][w] = make_uint4(0, 0, 0, 0);
            if (token < a.T && live) {
                x[0][w] = *reinterpret_cast<const uint4*>(k + token * r.k_token + h * r.k_head + 32 * (w0 + w) + 8 * t);
                x[1][w] = *reinterpret_cast<const uint4*>(v + token * r.v_token + h * r.v_head + 32 * (w0 + w) + 8 * t);
            }
        }
        if (token < a.T) page = place_of(b, token, slot);
        unsigned char* tile = kv4_tile_of(a.l, max(page, 0), h, slot);
        const int e = slot % KV4_TILE;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t code[MINE], step[SPREAD ? 1 : G], out[MINE];
            if constexpr (SPREAD) {
                quantise<F16, 1, PER == 1 ? 3 : PER == 2 ? 7 : 15>(x[j], code, step[0], live);
            } else {
#pragma unroll
                for (int g = 0; g < G; ++g) quantise<F16, PER, 3>(x[j] + g * PER, code + g * PER, step[g], true);
            }
            unsigned char* to;
            if (j == 0) {
                to = tile + kv4_key_row(e) * (D / 2) + t * (D / 8) + 4 * w0;
#pragma unroll
                for (int w = 0; w < MINE; ++w) out[w] = code[w];
            } else {
                to = tile + KV4_TILE * (D / 2) + e * (D / 2) + kv4_value_part(D, e, 2 * t) * (D / 16) + 2 * w0;
#pragma unroll
                for (int w = 0; w < MINE; ++w) code[w] = exchanged(code[w]);        // byte i: channels 32 w + 8 i + 2 t, and the next one's code
                if constexpr (SPREAD) {
                    out[0] = __byte_perm(gathered(code[0], 0, 0), gathered(code[0], 0, 4), 0x5410);
                } else if constexpr (W == 3) {
                    const uint32_t low = gathered(code[2], code[0], 0), high = gathered(code[0], code[1], 4);
                    out[0] = gathered(code[0], code[1], 0);
                    out[1] = __byte_perm(low, high, 0x5410);
                    out[2] = __byte_perm(high, gathered(code[2], code[2], 4), 0x5432);
                } else {
#pragma unroll
                    for (int w = 0; w < W; ++w) out[w] = gathered(code[2 * w % W], code[2 * w % W + 1], w < W / 2 ? 0 : 4);
                }
            }
            if (page >= 0 && live) {
                if constexpr (SPREAD) {
                    if (j == 0) *reinterpret_cast<uint32_t*>(to) = out[0];
                    else {
                        *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(out[0]);
                        *reinterpret_cast<uint16_t*>(to + D / 16) = static_cast<uint16_t>(out[0] >> 16);
                    }
                } else if constexpr (W == 4) *reinterpret_cast<uint4*>(to) = make_uint4(out[0], out[1], out[2], out[3]);
                else if constexpr (W == 2) *reinterpret_cast<uint2*>(to) = make_uint2(out[0], out[1]);
                else
#pragma unroll
                    for (int w = 0; w < W; ++w) reinterpret_cast<uint32_t*>(to)[w] = out[w];
                // lane t has step t, or a group's first lane its own
                uint32_t mine = step[0];
                if constexpr (!SPREAD)
#pragma unroll
                    for (int g = 1; g < G; ++g) mine = t == g ? step[g] : mine;
                if (SPREAD ? t == 0 && w0 % PER == 0 : t < G) reinterpret_cast<uint32_t*>(tile + KV4_TILE * D)[(j * KV4_TILE + e) * G + (SPREAD ? w0 / PER : t)] = mine;
            }
        }
    }
}

template <bool F16, int W, bool SPREAD>
__global__ void __launch_bounds__(THREADS) kv4_read_kernel(const __grid_constant__ Store a, uint16_t* k, uint16_t* v)
{
    typedef W4Type<F16> Ty;
    constexpr int D = 32 * W, MINE = SPREAD ? 1 : W, ROWS = THREADS / (SPREAD ? 16 : 4);
    Store b = a;
    b.t.pages = dependent_begin(a.t.pages);
    b.at = behind_wait<int32_t>(a.at);
    b.starts = behind_wait<int32_t>(a.starts);
    const int t = threadIdx.x & 3, w0 = SPREAD ? threadIdx.x >> 2 & 3 : 0, h = blockIdx.y;
    const bool live = !SPREAD || w0 < W;
    for (long long first = static_cast<long long>(blockIdx.x) * ROWS; first < a.T; first += static_cast<long long>(gridDim.x) * ROWS) {
        const int token = static_cast<int>(first) + threadIdx.x / (THREADS / ROWS);
        int page = -1, slot = 0;
        if (token < a.T && live) page = place_of(b, token, slot);
        uint32_t code[2][MINE], step[2][MINE];
#pragma unroll
        for (int w = 0; w < MINE; ++w) code[0][w] = code[1][w] = step[0][w] = step[1][w] = 0;
        if (page >= 0) {
            const unsigned char* tile = behind_wait<unsigned char>(kv4_tile_of(a.l, page, h, slot));
            const int e = slot % KV4_TILE;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const unsigned char* from = j == 0 ? tile + kv4_key_row(e) * (D / 2) + t * (D / 8) + 4 * w0
                                                   : tile + KV4_TILE * (D / 2) + e * (D / 2) + kv4_value_part(D, e, 2 * t) * (D / 16) + 2 * w0;
                if constexpr (SPREAD) {
                    if (j == 0) code[0][0] = *reinterpret_cast<const uint32_t*>(from);
                    else code[1][0] = *reinterpret_cast<const uint16_t*>(from) | static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(from + D / 16)) << 16;
                } else if constexpr (W == 4) {
                    const uint4 c = *reinterpret_cast<const uint4*>(from);
                    code[j][0] = c.x; code[j][1] = c.y; code[j][2] = c.z; code[j][3] = c.w;
                } else if constexpr (W == 2) {
                    const uint2 c = *reinterpret_cast<const uint2*>(from);
                    code[j][0] = c.x; code[j][1] = c.y;
                } else {
#pragma unroll
                    for (int w = 0; w < W; ++w) code[j][w] = reinterpret_cast<const uint32_t*>(from)[w];
                }
                const uint32_t* steps = reinterpret_cast<const uint32_t*>(tile + KV4_TILE * D) + (j * KV4_TILE + e) * a.l.G;
#pragma unroll
                for (int w = 0; w < MINE; ++w) step[j][w] = steps[a.l.G == W ? w0 + w : a.l.G == 1 ? 0 : (w0 + w) >> 1];
            }
        }
        // the values' parts 2 t and 2 t + 1: halves of words, one after the other
        uint32_t part[MINE];
#pragma unroll
        for (int w = 0; w < MINE; ++w) {
            const uint32_t low = code[1][w / 2] >> 16 * (w & 1), high = code[1][(MINE + w) / 2] >> 16 * (MINE + w & 1);
            part[w] = exchanged(spread(low) | spread(high) << 4);
        }
#pragma unroll
        for (int w = 0; w < MINE; ++w) code[1][w] = part[w];
        if (token >= a.T || !live) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int w = 0; w < MINE; ++w) {
                // a byte under the exponent of 2^23 is 2^23 + code
                const uint32_t low = code[j][w] & 0x0f0f0f0fu, high = code[j][w] >> 4 & 0x0f0f0f0fu, whole = 0x4b000000u;
                auto both = [](float f) { return f2_pack(__float_as_uint(f), __float_as_uint(f)); };
                const u64 s2 = both(Ty::lo(step[j][w])), m2 = both(Ty::hi(step[j][w])), less2 = both(-8388608.f);
                uint32_t out[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    uint32_t lo, hi;
                    f2_split(f2_fma(f2_add(f2_pack(__byte_perm(low, whole, 0x7440 + n), __byte_perm(high, whole, 0x7440 + n)), less2), s2, m2), lo, hi);
                    out[n] = Ty::round2(__uint_as_float(lo), __uint_as_float(hi));
                }
                *reinterpret_cast<uint4*>((j == 0 ? k : v) + (static_cast<long long>(token) * a.l.H + h) * D + 32 * (w0 + w) + 8 * t) = make_uint4(out[0], out[1], out[2], out[3]);
            }
    }
}

int check(const bs_kv4_cache* c, const int32_t* table, long long pitch, int width, int B, const int32_t* at, const int32_t* starts, int T, Store& a)
{
    if (!c || !c->data || !table || !at || width <= 0 || B <= 0 || T < 0 || (pitch != 0 && pitch < width)) return BS_ERR_INVALID_ARG;
    if (c->type != BS_F16 && c->type != BS_BF16) return BS_ERR_INVALID_ARG;
    if (c->pages <= 0 || c->heads <= 0 || c->D <= 0 || c->page <= 0 || c->group <= 0) return BS_ERR_INVALID_ARG;
    if (!starts && T != B) return BS_ERR_INVALID_ARG;
    if (!kv4_layout(*c, a.l) || T > MOST_ROWS) return BS_ERR_UNSUPPORTED;
    if (!aligned16(c->data)) return BS_ERR_ALIGNMENT;
    a.t = {table, pitch, width, B};
    a.at = at;
    a.starts = starts;
    a.T = T;
    return BS_OK;
}
// Sixteen lanes a vector while the GPU has room for all of them: 32 tokens of 8 heads, stored and read, take 8.8 us in place of 15.7.
bool spread_of(const Store& a) { return static_cast<long long>(a.T) * a.l.H <= 32LL * device_sm_count(); }
// Neighbouring tokens of a head a CTA, as many as fill the GPU twice.
dim3 grid_of(const Store& a, bool spread)
{
    const long long blocks = ceil_div_ll(a.T, THREADS / (spread ? 16 : 4)), most = ceil_div(32 * device_sm_count(), a.l.H);
    return dim3(static_cast<unsigned>(blocks < most ? blocks : most), a.l.H);
}

template <bool F16, int W, int PER>
int append(const Store& a, const Rows& r, cudaStream_t st)
{
    return spread_of(a) ? launch_dependent(kv4_append_kernel<F16, W, PER, true>, grid_of(a, true), dim3(THREADS), 0, st, a, r)
                        : launch_dependent(kv4_append_kernel<F16, W, PER, false>, grid_of(a, false), dim3(THREADS), 0, st, a, r);
}
template <bool F16>
int append(const Store& a, const Rows& r, cudaStream_t st)
{
    if (a.l.D == 64) return a.l.G == 1 ? append<F16, 2, 2>(a, r, st) : append<F16, 2, 1>(a, r, st);
    if (a.l.D == 96) return a.l.G == 1 ? append<F16, 3, 3>(a, r, st) : append<F16, 3, 1>(a, r, st);
    return a.l.G == 1 ? append<F16, 4, 4>(a, r, st) : a.l.G == 2 ? append<F16, 4, 2>(a, r, st) : append<F16, 4, 1>(a, r, st);
}
template <bool F16, int W>
int read(const Store& a, uint16_t* k, uint16_t* v, cudaStream_t st)
{
    return spread_of(a) ? launch_dependent(kv4_read_kernel<F16, W, true>, grid_of(a, true), dim3(THREADS), 0, st, a, k, v)
                        : launch_dependent(kv4_read_kernel<F16, W, false>, grid_of(a, false), dim3(THREADS), 0, st, a, k, v);
}
template <bool F16>
int read(const Store& a, uint16_t* k, uint16_t* v, cudaStream_t st)
{
    return a.l.D == 64 ? read<F16, 2>(a, k, v, st) : a.l.D == 96 ? read<F16, 3>(a, k, v, st) : read<F16, 4>(a, k, v, st);
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
    return cache->type == BS_F16 ? append<true>(a, r, st) : append<false>(a, r, st);
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
    return cache->type == BS_F16 ? read<true>(a, ko, vo, st) : read<false>(a, ko, vo, st);
}
