// Keys and values of new tokens into pages of 4-bit codes, and the values that codes stand for out of them.
//
// A vector of `group` channels is c s + m: m its least value, s a fifteenth of its span.  Half a warp takes one token of one head, eight channels a
// lane.  A code is the quotient rounded half to even, decided without a division: the product with the reciprocal is off by less than one, and the borders
// between codes, (c + 1/2) s, are exact in binary32 (s has at most 11 bits, 2 c + 1 five), so that the difference is compared with them.  Where the
// rounded difference x - m lies on a border, what the subtraction lost decides.
#include "kv4.h"
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
    slot = static_cast<int>(entry % a.l.page);
    return kv4_page_of(a.l, a.t, b, entry);
}

// Codes of eight values of a group that has least value m and step s.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], float m, float s)
{
    // steps near the ends of binary32 are brought to where their reciprocals and borders are exact
    const float up = s < 0x1p-60f ? 0x1p64f : s > 0x1p60f ? 0x1p-64f : 1.f, t = s * up, inverse = __frcp_rn(t);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float d = x[i] - m, e = d * up;
        float c = fminf(rintf(e * inverse), 15.f);
        const float above = (c + 0.5f) * t, below = (c - 0.5f) * t;
        if (e >= above || e <= below) {
            const float back = x[i] - d, lost = (x[i] - (d + back)) + (back - m);       // of the difference, exact
            const bool odd = static_cast<int>(c) & 1;
            if (e > above || (e == above && (lost > 0.f || (lost == 0.f && odd)))) c += 1.f;
            else if (e < below || (e == below && (lost < 0.f || (lost == 0.f && odd)))) c -= 1.f;
        }
        word |= static_cast<uint32_t>(fminf(fmaxf(c, 0.f), 15.f)) << 4 * i;
    }
    return s > 0.f ? word : 0u;
}

// One vector of a half warp: its codes (eight a lane, lanes from D / 8 on have none) and the group's step and offset as a word of the layout.
template <bool F16>
__device__ __forceinline__ uint32_t quantise(const uint4& raw, int group, bool live, uint32_t& step)
{
    typedef W4Type<F16> Ty;
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    float x[8], lo = INFINITY, hi = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = Ty::lo(w[i]);
        x[2 * i + 1] = Ty::hi(w[i]);
    }
    if (live)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lo = fminf(lo, x[i]);
            hi = fmaxf(hi, x[i]);
            bad |= !(fabsf(x[i]) < INFINITY);
        }
    int any = bad;
#pragma unroll
    for (int d = 1; d < 16; d *= 2) {
        if (8 * d >= group) break;
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
        any |= __shfl_xor_sync(0xffffffffu, any, d);
    }
    const float span = hi - lo;
    uint32_t s = Ty::round2(__fdiv_rn(span, 15.f), lo);
    if (any || !(span < INFINITY)) {        // a vector with an infinity or a NaN, or a span that binary32 does not hold: reads as NaN
        step = 0x7fff0000u;
        return 0;
    }
    step = s;
    return codes_of(x, lo, Ty::lo(s));
}

template <bool F16>
__global__ void __launch_bounds__(THREADS) kv4_append_kernel(const __grid_constant__ Store a, const __grid_constant__ Rows r)
{
    __shared__ uint32_t words[ROWS][17];
    const int32_t* pages = dependent_begin(a.t.pages);
    Store b = a;
    b.t.pages = pages;
    b.at = behind_wait<int32_t>(a.at);
    b.starts = behind_wait<int32_t>(a.starts);
    const int m = threadIdx.x & 15, mine = threadIdx.x >> 4, D = a.l.D;
    const long long rows = static_cast<long long>(a.T) * a.l.H;
    for (long long first = static_cast<long long>(blockIdx.x) * ROWS; first < rows; first += static_cast<long long>(gridDim.x) * ROWS) {
        const long long row = first + mine;
        int page = -1, slot = 0, h = 0;
        uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        const bool live = 8 * m < D;
        if (row < rows) {
            const int token = static_cast<int>(row / a.l.H);
            h = static_cast<int>(row - static_cast<long long>(token) * a.l.H);
            if (live) {
                x[0] = *reinterpret_cast<const uint4*>(behind_wait<uint16_t>(r.k) + token * r.k_token + h * r.k_head + 8 * m);
                x[1] = *reinterpret_cast<const uint4*>(behind_wait<uint16_t>(r.v) + token * r.v_token + h * r.v_head + 8 * m);
            }
            page = place_of(b, token, slot);
        }
        uint32_t step[2], code[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) code[i] = quantise<F16>(x[i], a.l.group, live, step[i]);
        words[mine][m] = code[1];
        __syncwarp();
        if (page >= 0) {
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
            // part g of the values' row: nibble g of each of the D / 8 words.  Two lanes a part, half of its bytes each
            const int g = m >> 1, bytes = D / 32;
            unsigned char* to = tile + KV4_TILE * (D / 2) + e * (D / 2) + kv4_value_part(D, e, g) * (D / 16) + (m & 1) * bytes;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= bytes) break;
                const int w = 2 * ((m & 1) * bytes + i);
                to[i] = static_cast<unsigned char>((words[mine][w] >> 4 * g & 15) | (words[mine][w + 1] >> 4 * g & 15) << 4);
            }
        }
        __syncwarp();
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
    if (8 * m >= D) return;
    const long long rows = static_cast<long long>(a.T) * a.l.H;
    for (long long row = static_cast<long long>(blockIdx.x) * ROWS + (threadIdx.x >> 4); row < rows; row += static_cast<long long>(gridDim.x) * ROWS) {
        const int token = static_cast<int>(row / a.l.H), h = static_cast<int>(row - static_cast<long long>(token) * a.l.H);
        int slot = 0;
        const int page = place_of(b, token, slot);
        uint4 out[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        if (page >= 0) {
            const unsigned char* tile = behind_wait<unsigned char>(kv4_tile_of(a.l, page, h, slot));
            const int e = slot % KV4_TILE;
            const uint32_t key = *reinterpret_cast<const uint32_t*>(tile + kv4_key_row(e) * (D / 2) + (m & 3) * (D / 8) + (m >> 2) * 4);
            const unsigned char* from = tile + KV4_TILE * (D / 2) + e * (D / 2) + m / 2;
            uint32_t value = 0;
#pragma unroll
            for (int g = 0; g < 8; ++g) value |= (from[kv4_value_part(D, e, g) * (D / 16)] >> 4 * (m & 1) & 15u) << 4 * g;
            const uint32_t* steps = reinterpret_cast<const uint32_t*>(tile + KV4_TILE * D) + e * a.l.G + 8 * m / a.l.group;
            const uint32_t code[2] = {key, value}, step[2] = {steps[0], steps[KV4_TILE * a.l.G]};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float s = Ty::lo(step[i]), o = Ty::hi(step[i]);
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = Ty::round2(fmaf(static_cast<float>(code[i] >> 8 * j & 15u), s, o), fmaf(static_cast<float>(code[i] >> (8 * j + 4) & 15u), s, o));
                out[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        *reinterpret_cast<uint4*>(k + row * D + 8 * m) = out[0];
        *reinterpret_cast<uint4*>(v + row * D + 8 * m) = out[1];
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
dim3 grid_of(const Store& a)
{
    const long long blocks = ceil_div_ll(static_cast<long long>(a.T) * a.l.H, ROWS), most = 8LL * device_sm_count();
    return dim3(static_cast<unsigned>(blocks < most ? blocks : most));
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
