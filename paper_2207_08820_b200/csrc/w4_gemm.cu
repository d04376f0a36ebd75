// Product of 16-bit activations with 4-bit weights: y[m][o] = sum_g s[o][g] * sum_{k in g} x[m][k] (q[o][k] - z[o][g]) + bias[o].
//
// Few rows of x: bound by the weights' bytes.  w4_gemm_kernel streams them through shared memory, every warp a part of the reduction of 16 rows, and
// multiplies with mma.sync (w4_dot.cuh), where eight rows of x cost what one does; products are exact, sums of a group in 32 bits, scaled in
// 32 bits, and rounded once.
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int WARPS = 8, STAGES = 6;

// An item is 16 rows of the weights and 8 NT rows of x.  `split` warps of a CTA share an item's reduction, block by block in turn; a CTA works on
// WARPS / split items at a time and goes on to others, whose blocks are on their way while the sums of the current ones are put together.
template <bool F16, int NG, bool ZEROS, int NT>
__global__ void __launch_bounds__(WARPS * 32, 2) w4_gemm_kernel(const __grid_constant__ W4Gemm g, int split)
{
    typedef typename W4Type<F16>::T T;
    typedef W4Stage<NG, ZEROS> Stage;
    extern __shared__ __align__(16) unsigned char ring[];      // [WARPS][STAGES] stages
    __shared__ float part[WARPS][NT * 8][17];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, m0 = blockIdx.y * NT * 8;
    const int side = WARPS / split, sub = warp / split, k0 = warp % split;
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(ring)) + warp * STAGES * Stage::BYTES;
    const unsigned char* w = dependent_begin(g.w);
    // the blocks that this warp copies, STAGES - 1 ahead of the ones it multiplies
    int crb = blockIdx.x * side + sub, ccb = k0, cslot = 0;
    const bool some = k0 < g.l.cbs;
    auto copy = [&] {
        if (some && crb < g.l.rbs) {
            Stage::copy(mine + cslot * Stage::BYTES, w, g.l, crb, ccb, lane);
            ccb += split;
            if (ccb >= g.l.cbs) { ccb = k0; crb += gridDim.x * side; }
        }
        ring_commit();
        cslot = cslot + 1 == STAGES ? 0 : cslot + 1;
    };
#pragma unroll 1
    for (int s = 0; s < STAGES - 1; ++s) copy();
    int slot = 0;
    for (int first = blockIdx.x * side; first < g.l.rbs; first += gridDim.x * side) {
        const int rb = first + sub;
        float tot[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) tot[n][0] = tot[n][1] = tot[n][2] = tot[n][3] = 0.f;
        if (rb < g.l.rbs) {
            for (int cb = k0; cb < g.l.cbs; cb += split) {
                uint4 x[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int m = m0 + n * 8 + (lane >> 2);
                    const T* row = static_cast<const T*>(g.x) + m * g.ldx;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[n][j] = m < g.M ? load_x(row, cb * 128 + 32 * j + 8 * (lane & 3), g.l.K) : make_uint4(0, 0, 0, 0);
                }
                ring_wait<STAGES - 2>();
                W4Tile<NG, ZEROS> tile;
                tile.take(mine + slot * Stage::BYTES, g.l, cb, lane);
                slot = slot + 1 == STAGES ? 0 : slot + 1;
                copy();     // into the stage before this one, which every lane has read: the warp met in ring_wait since
                w4_block<F16, F16, NG, ZEROS, NT>(tile, x, tot);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int m = n * 8 + 2 * (lane & 3), r = lane >> 2;
            part[warp][m][r] = tot[n][0];
            part[warp][m + 1][r] = tot[n][1];
            part[warp][m][r + 8] = tot[n][2];
            part[warp][m + 1][r + 8] = tot[n][3];
        }
        __syncthreads();
        // the warps' parts are added in their order: the same bits every time
        for (int i = threadIdx.x; i < side * NT * 8 * 16; i += WARPS * 32) {
            const int q = i / (NT * 8 * 16), m = (i >> 4) % (NT * 8), r = i & 15, o = (first + q) * 16 + r;
            if (m0 + m >= g.M || o >= g.l.O) continue;
            float v = 0.f;
            for (int k = 0; k < split; ++k) v += part[q * split + k][m][r];
            if (g.bias) v += static_cast<float>(static_cast<const T*>(g.bias)[o]);
            static_cast<T*>(g.y)[(m0 + m) * g.ldy + o] = W4Type<F16>::round(v);
        }
        __syncthreads();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// Rows of x that do not start on 16-byte boundaries, brought to ones that do, zeros behind K.
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
    const size_t smem = WARPS * STAGES * W4Stage<NG, ZEROS>::BYTES;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess) { cudaGetLastError(); return BS_ERR_CUDA; }
    int split = WARPS;
    while (split > 1 && split / 2 >= g.l.cbs) split /= 2;
    const int ctas = ceil_div(g.l.rbs, WARPS / split);
    return launch_dependent(kernel, dim3(ctas < 2 * sms ? ctas : 2 * sms, ceil_div(g.M, 8 * NT)), dim3(WARPS * 32), smem, st, g, split);
}
template <bool F16, int NG, bool ZEROS>
int launch_rows(const W4Gemm& g, int sms, cudaStream_t st)
{
    if (g.M <= 8) return launch_tile<F16, NG, ZEROS, 1>(g, sms, st);
    if (g.M <= 16) return launch_tile<F16, NG, ZEROS, 2>(g, sms, st);
    return launch_tile<F16, NG, ZEROS, 4>(g, sms, st);
}
template <bool F16>
int launch(const W4Gemm& g, int sms, cudaStream_t st)
{
    const int ng = g.l.group == 32 ? 4 : g.l.group == 64 ? 2 : 1;
    if (g.l.zeros) return ng == 4 ? launch_rows<F16, 4, true>(g, sms, st) : ng == 2 ? launch_rows<F16, 2, true>(g, sms, st) : launch_rows<F16, 1, true>(g, sms, st);
    return ng == 4 ? launch_rows<F16, 4, false>(g, sms, st) : ng == 2 ? launch_rows<F16, 2, false>(g, sms, st) : launch_rows<F16, 1, false>(g, sms, st);
}

bool rows_aligned(int M, long long ldx) { return M == 1 || ldx % 8 == 0; }

}  // namespace
}  // namespace bs

extern "C" size_t bs_w4_gemm_workspace_bytes(int M, int K, long long ldx)
{
    if (M <= 0 || K <= 0 || bs::rows_aligned(M, ldx)) return 0;
    return static_cast<size_t>(M) * ((static_cast<size_t>(K) + 7) & ~static_cast<size_t>(7)) * 2;
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
    if (!rows_aligned(M, ldx) && (!workspace || workspace_bytes < bs_w4_gemm_workspace_bytes(M, K, ldx))) return BS_ERR_INVALID_ARG;
    const int sms = device_sm_count();
    if (sms <= 0) return BS_ERR_CUDA;
    if (!rows_aligned(M, ldx)) {
        const int ldo = (K + 7) & ~7;
        const long long want = (static_cast<long long>(M) * (ldo / 8) + 255) / 256, most = static_cast<long long>(sms) * 8;
        const int rc = launch_dependent(w4_align_rows_kernel, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(256), 0, st,
                                        static_cast<const uint16_t*>(x), ldx, M, K, static_cast<uint16_t*>(workspace), ldo);
        if (rc != BS_OK) return rc;
        g.x = workspace;
        g.ldx = ldo;
    }
    return type == BS_F16 ? launch<true>(g, sms, st) : launch<false>(g, sms, st);
}
