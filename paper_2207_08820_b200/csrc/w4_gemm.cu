// Product of 16-bit activations with 4-bit weights: y[m][o] = sum_g s[o][g] * sum_{k in g} x[m][k] (q[o][k] - z[o][g]) + bias[o].
//
// Few rows of x: w4_gemm_kernel streams the weights through shared memory, every warp a part of the reduction of 16 rows, and multiplies with mma.sync
// (w4_dot.cuh), where eight rows of x cost what one does; products are exact, sums of a group in 32 bits, scaled in 32 bits, and rounded once.
// The bytes of the weights would bound it; what does is the expansion of the codes, whose instructions fill 60 % of the issue slots, the rest waits for
// one another.  One row, 24576 x 8192: 28.7 us, 3.6 TB/s, where the bare stream takes 18 and the copy rate 16 (with 8 rows 31, with 16 46).  More rows:
// csrc/w4_mma.cu.
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int WARPS = 8, STAGES = 6;

// An item is 16 rows of the weights for each of WARPS / split teams and 8 NT rows of x; a team's warps take the blocks of the reduction in turn.  A CTA goes
// through several items; the last warp copies their blocks ahead, also while the sums of an item are put together.
// Per SM, as the registers allow: a fourth CTA of one tile spills (1 x 4096 x 4096 6.4 us in place of 5.3).
template <int NT> constexpr int ctas_of() { return NT == 1 ? 3 : 2; }
template <bool F16, int NG, bool ZEROS, int NT>
__global__ void __launch_bounds__(WARPS * 32 + 32, ctas_of<NT>()) w4_gemm_kernel(const __grid_constant__ W4Gemm g, const __grid_constant__ CUtensorMap tw, int split)
{
    typedef typename W4Type<F16>::T T;
    constexpr int M = NT * 8;
    // whole blocks in a loop of their own, where the registers hold what both loops keep: one row, 4096 x 4096, 4.9 in place of 5.3 us; with zero points 8 rows of
    // 16384 x 4096 would take 16.2 in place of 14.1, two tiles of x 21 in place of 15.5 (16 rows, 4096 x 16384)
    constexpr bool OWN = NT == 1 && !ZEROS;
    typedef W4TeamRing<NG, ZEROS, 1, WARPS, STAGES> Ring;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[2 * STAGES];
    __shared__ float parts[2][WARPS][M][17];        // items take turns: one barrier each
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, m0 = blockIdx.y * M;
    const int teams = WARPS / split, team = warp / split, k0 = warp % split;
    Ring ring(smem, bars, warp, lane);
    // the first stages' blocks start for L2 while the kernel in front drains: products in a row, one row of x, take 5.6 in place of 6.2 us each
    // (4096 x 4096), 13.0 in place of 15.0 (8192 x 8192)
    if (warp == WARPS && lane == 0)
        for (int c = 0; c < g.l.cbs && c < STAGES * split; c += split) Ring::hint(&tw, blockIdx.x * teams, c, 0);
    dependent_begin(g.w);
    if (warp == WARPS) {
        const CUtensorMap* const maps[1] = {&tw};
        if (lane == 0) {
            int filled = 0;
            for (int rb0 = blockIdx.x * teams; rb0 < g.l.rbs; rb0 += gridDim.x * teams)
                for (int c = 0; c < g.l.cbs; c += split, ++filled) ring.fill(maps, {rb0}, c, 0, g.status);
            ring.drain(filled, g.status);
        }
        return;
    }
    const T* x0 = behind_wait<T>(g.x);
    const T* row[NT];       // lanes without a row of x compute the last one's again
#pragma unroll
    for (int n = 0; n < NT; ++n) row[n] = x0 + min(m0 + n * 8 + (lane >> 2), g.M - 1) * g.ldx + 8 * (lane & 3);
    const int full = g.l.K / W4_COLS;
    float tot[1][NT][4];
    // One turn: block c of the team's rows.  whole: it lies before K.
    auto turn_of = [&](int c, bool whole) {
        uint4 x[NT][4];
        if (whole || c < g.l.cbs) {
#pragma unroll
            for (int n = 0; n < NT; ++n) load_block_x(x[n], row[n], c, g.l.K, whole, lane);
        }
        ring.landed(g.status);
        if (whole || c < g.l.cbs) {
            W4Tile<NG, ZEROS> w[1];
            ring.take(w);
            w4_blocks<F16, F16, 1>(w, [&](int n, int j, int) { return x[n][j]; }, tot);
        }
        ring.release(lane);
        ring.next();
    };
    int turn = 0;
    for (int rb0 = blockIdx.x * teams; rb0 < g.l.rbs; rb0 += gridDim.x * teams, turn ^= 1) {
        float (*part)[M][17] = parts[turn];
        const int rb = rb0 + team;
#pragma unroll
        for (int n = 0; n < NT; ++n) tot[0][n][0] = tot[0][n][1] = tot[0][n][2] = tot[0][n][3] = 0.f;
        // teams without rows multiply what the stages hold, and drop it
        int c = k0;
        if (OWN)
            for (; c < full; c += split) turn_of(c, true);
        for (; c < g.l.cbs + k0; c += split) turn_of(c, !OWN && c < full);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[warp][n * 8 + 2 * (lane & 3) + (i & 1)][(lane >> 2) + 8 * (i >> 1)] = tot[0][n][i];
        asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 * split) : "memory");
        // the warps' parts are added in their order: the same bits every time
        for (int i = k0 * 32 + lane; i < M * 16; i += split * 32) {
            const int m = i >> 4, r = i & 15, o = rb * W4_ROWS + r;
            if (m0 + m >= g.M || o >= g.l.O) continue;
            float v = 0.f;
            for (int k = 0; k < split; ++k) v += part[team * split + k][m][r];
            v *= W4Type<F16>::PART;
            if (g.bias) v += static_cast<float>(static_cast<const T*>(g.bias)[o]);
            static_cast<T*>(g.y)[(m0 + m) * g.ldy + o] = W4Type<F16>::round(v);
        }
    }
}

// Rows of x that do not start on 16-byte boundaries, brought to ones that do, zeros behind K: the products' loads and tensor copies are of 16 bytes.  One more
// launch, 2.9 us with 33 rows of 4611 columns (1383 outputs: 10.5 in place of 7.6 us), bound by its latency and by the host; 1.7 us in a graph (8 rows of 4097).
__global__ void __launch_bounds__(256) w4_align_rows_kernel(const uint16_t* x, long long ldx, int M, int K, uint16_t* out, int ldo)
{
    x = dependent_begin(x);
    const int chunks = ldo / 8;
    const long long step = static_cast<long long>(gridDim.x) * blockDim.x;
    for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < static_cast<long long>(M) * chunks; i += step) {
        const int m = static_cast<int>(i / chunks), k0 = static_cast<int>(i - static_cast<long long>(m) * chunks) * 8;
        uint32_t e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = k0 + k < K ? x[m * ldx + k0 + k] : 0;
        *reinterpret_cast<uint4*>(out + static_cast<long long>(m) * ldo + k0) = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    }
}

template <bool F16, int NG, bool ZEROS, int NT>
int launch_tile(const W4Gemm& g, int sms, cudaStream_t st)
{
    auto kernel = w4_gemm_kernel<F16, NG, ZEROS, NT>;
    constexpr int smem = W4TeamRing<NG, ZEROS, 1, WARPS, STAGES>::BYTES;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) { cudaGetLastError(); return BS_ERR_CUDA; }
    const int places = ctas_of<NT>() * sms;
    const int split = w4_team_width(WARPS, g.l.cbs);
    const int items = ceil_div(g.l.rbs, WARPS / split), tiles = ceil_div(g.M, 8 * NT);
    CUtensorMap tw;
    if (!w4_encode_blocks(&tw, g.w, g.l, 1, split, WARPS / split)) return BS_ERR_CUDA;
    return launch_dependent(kernel, dim3(items < places ? items : places, tiles), dim3(WARPS * 32 + 32), smem, st, g, tw, split);
}
template <bool F16, int NG, bool ZEROS>
int launch_tiles(const W4Gemm& g, int sms, cudaStream_t st)
{
    // a tile of 16 rows costs more than one of 8 (24576 x 8192: 9 rows 41 us, 8 rows 31) and less than two of them, which would read the weights twice
    return g.M <= 8 ? launch_tile<F16, NG, ZEROS, 1>(g, sms, st) : launch_tile<F16, NG, ZEROS, 2>(g, sms, st);
}
template <bool F16>
int launch(const W4Gemm& g, int sms, cudaStream_t st)
{
    const int ng = g.l.group == 32 ? 4 : g.l.group == 64 ? 2 : 1;
    if (g.l.zeros) return ng == 4 ? launch_tiles<F16, 4, true>(g, sms, st) : ng == 2 ? launch_tiles<F16, 2, true>(g, sms, st) : launch_tiles<F16, 1, true>(g, sms, st);
    return ng == 4 ? launch_tiles<F16, 4, false>(g, sms, st) : ng == 2 ? launch_tiles<F16, 2, false>(g, sms, st) : launch_tiles<F16, 1, false>(g, sms, st);
}

bool rows_aligned(int M, long long ldx) { return M == 1 || ldx % 8 == 0; }

}  // namespace
}  // namespace bs

namespace bs {
namespace {
size_t aligned_bytes(int M, int K, long long ldx) { return rows_aligned(M, ldx) ? 0 : static_cast<size_t>(M) * ((static_cast<size_t>(K) + 7) & ~static_cast<size_t>(7)) * 2; }
int sm_count()
{
    const int sms = device_sm_count();
    return sms > 0 ? sms : 148;     // a query without a device plans for a full B200
}
}  // namespace
}  // namespace bs

extern "C" size_t bs_w4_gemm_workspace_bytes(int M, int O, int K, int group, long long ldx)
{
    using namespace bs;
    W4Layout l;
    if (M <= 0 || M > W4_MAX_DIM || !w4_layout(O, K, group, 0, l)) return 0;
    const int sms = sm_count();
    return aligned_bytes(M, K, ldx) + (w4_mma_wanted(M, l, sms) ? w4_mma_workspace(M, l, sms) : 0);
}

extern "C" int bs_w4_gemm(const void* x, long long ldx, int M, const void* w, int O, int K, int group, int zeros, bs_float_t type, const void* bias, void* y,
                          long long ldy, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace bs;
    W4Gemm g{};
    if (!x || !w || !y || M < 0 || O <= 0 || K <= 0 || group <= 0 || ldx < K || ldy < O || (type != BS_F16 && type != BS_BF16)) return BS_ERR_INVALID_ARG;
    if (M > W4_MAX_DIM || !w4_layout(O, K, group, zeros, g.l)) return BS_ERR_UNSUPPORTED;
    if (!aligned16(x) || !aligned16(w) || !aligned16(bias) || !aligned16(y) || !aligned16(workspace)) return BS_ERR_ALIGNMENT;
    if (M == 0) return BS_OK;
    g.x = x; g.w = static_cast<const unsigned char*>(w); g.bias = bias; g.y = y; g.ldx = ldx; g.ldy = ldy; g.M = M;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const size_t need = bs_w4_gemm_workspace_bytes(M, O, K, group, ldx);
    if (need && (!workspace || workspace_bytes < need)) return BS_ERR_INVALID_ARG;
    const int sms = device_sm_count();
    g.status = status_device_ptr();
    if (sms <= 0 || !g.status) return BS_ERR_CUDA;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    if (!rows_aligned(M, ldx)) {
        const int ldo = (K + 7) & ~7;
        const long long want = (static_cast<long long>(M) * (ldo / 8) + 255) / 256, most = static_cast<long long>(sms) * 8;
        const int rc = launch_dependent(w4_align_rows_kernel, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(256), 0, st,
                                        static_cast<const uint16_t*>(x), ldx, M, K, reinterpret_cast<uint16_t*>(ws), ldo);
        if (rc != BS_OK) return rc;
        g.x = ws;
        g.ldx = ldo;
        ws += aligned_bytes(M, K, ldx);
    }
    if (w4_mma_wanted(M, g.l, sms)) return w4_mma_launch(g, type == BS_F16, reinterpret_cast<float*>(ws), sms, st);
    return type == BS_F16 ? launch<true>(g, sms, st) : launch<false>(g, sms, st);
}
