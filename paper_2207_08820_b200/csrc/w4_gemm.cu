// Product of 16-bit activations with 4-bit weights: y[m][o] = sum_g s[o][g] * sum_{k in g} x[m][k] (q[o][k] - z[o][g]) + bias[o].
//
// Few rows of x: bound by the weights' bytes.  w4_gemm_kernel streams them through shared memory, every warp a part of the reduction of 16 rows, and
// multiplies with mma.sync (w4_dot.cuh), where eight rows of x cost what one does; products are exact, sums of a group in 32 bits, scaled in
// 32 bits, and rounded once.
#include <cstdlib>

#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int MOST_WARPS = 16;

// A CTA owns 16 RT rows of the weights and 8 NT rows of x; its warps take the blocks of the reduction in turn.
template <bool F16, int NG, bool ZEROS, int NT, int RT, int STAGES>
__global__ void __launch_bounds__(MOST_WARPS * 32, 1) w4_gemm_kernel(const __grid_constant__ W4Gemm g)
{
    typedef typename W4Type<F16>::T T;
    typedef W4Ring<NG, ZEROS, RT, STAGES> Ring;
    constexpr int M = NT * 8, R = RT * W4_ROWS, PITCH = R + 1;
    extern __shared__ __align__(128) unsigned char smem[];      // rings of the warps; in the end their sums, [warps][M][PITCH] floats
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, rb0 = blockIdx.x * RT, m0 = blockIdx.y * M;
    __shared__ uint64_t bars[MOST_WARPS][STAGES];
    Ring ring(smem, bars[warp], warp, lane);
    const unsigned char* from[RT];
    const unsigned char* matrix = dependent_begin(g.w);
    const T* x0 = behind_wait<T>(g.x);
#pragma unroll
    for (int r = 0; r < RT; ++r) from[r] = matrix + (static_cast<size_t>(min(rb0 + r, g.l.rbs - 1)) * g.l.cbs + warp) * Ring::BLOCK;
    int left = (g.l.cbs - warp + warps - 1) / warps;       // blocks that this warp has still to fetch
    auto put = [&] {
        if (left > 0) {
            ring.put(from, lane);
#pragma unroll
            for (int r = 0; r < RT; ++r) from[r] += warps * Ring::BLOCK;
            --left;
        }
    };
#pragma unroll 1
    for (int s = 0; s < STAGES - 1; ++s) put();
    const T* row[NT];       // lanes without a row of x compute the last one's again
#pragma unroll
    for (int n = 0; n < NT; ++n) row[n] = x0 + min(m0 + n * 8 + (lane >> 2), g.M - 1) * g.ldx;
    float tot[RT][NT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) tot[r][n][0] = tot[r][n][1] = tot[r][n][2] = tot[r][n][3] = 0.f;
    const int full = g.l.K / W4_COLS;
    for (int cb = warp; cb < g.l.cbs; cb += warps) {
        uint4 x[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) load_block_x(x[n], row[n], cb, g.l.K, cb < full, lane);
        W4Tile<NG, ZEROS> w[RT];
        ring.get(w, lane, g.status);
        put();      // into the stage before this one: its blocks have been multiplied
        w4_blocks<F16, F16, 1>(w, [&](int n, int j, int) { return x[n][j]; }, tot);
    }
    __syncthreads();
    float* part = reinterpret_cast<float*>(smem);
    float* mine = part + warp * M * PITCH;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(n * 8 + 2 * (lane & 3) + (i & 1)) * PITCH + r * W4_ROWS + (lane >> 2) + 8 * (i >> 1)] = tot[r][n][i];
        }
    __syncthreads();
    // the warps' parts are added in their order: the same bits every time
    for (int i = threadIdx.x; i < M * R; i += blockDim.x) {
        const int m = i / R, r = i % R, o = rb0 * W4_ROWS + r;
        if (m0 + m >= g.M || o >= g.l.O) continue;
        float v = 0.f;
        for (int k = 0; k < warps; ++k) v += part[(k * M + m) * PITCH + r];
        if (g.bias) v += static_cast<float>(static_cast<const T*>(g.bias)[o]);
        static_cast<T*>(g.y)[(m0 + m) * g.ldy + o] = W4Type<F16>::round(v);
    }
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

template <bool F16, int NG, bool ZEROS, int NT, int RT, int STAGES>
int launch_tile(const W4Gemm& g, int sms, cudaStream_t st)
{
    auto kernel = w4_gemm_kernel<F16, NG, ZEROS, NT, RT, STAGES>;
    const int items = ceil_div(g.l.rbs, RT), tiles = ceil_div(g.M, 8 * NT);
    // enough warps for 16 an SM, each with two blocks of the reduction at least
    int warps = MOST_WARPS;
    while (warps > 1 && (2 * warps > g.l.cbs + 1 || static_cast<long long>(items) * tiles * warps / 2 >= 16ll * sms)) warps /= 2;
#ifdef BS_TUNING
    if (const char* e = getenv("BS_W4_WARPS")) warps = atoi(e);
#endif
    const int ring = warps * W4Ring<NG, ZEROS, RT, STAGES>::BYTES, part = static_cast<int>(sizeof(float)) * warps * NT * 8 * (RT * W4_ROWS + 1);
    const int smem = ring > part ? ring : part;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) { cudaGetLastError(); return BS_ERR_CUDA; }
    return launch_dependent(kernel, dim3(items, tiles), dim3(warps * 32), smem, st, g);
}
template <bool F16, int NG, bool ZEROS>
int launch_rows(const W4Gemm& g, int sms, cudaStream_t st)
{
#ifdef BS_TUNING
    if (const char* e = getenv("BS_W4_RT")) {
        const int rt = atoi(e);
        if (g.M <= 8) return rt == 1 ? launch_tile<F16, NG, ZEROS, 1, 1, 8>(g, sms, st) : launch_tile<F16, NG, ZEROS, 1, 2, 6>(g, sms, st);
        if (g.M <= 16) return rt == 1 ? launch_tile<F16, NG, ZEROS, 2, 1, 8>(g, sms, st) : launch_tile<F16, NG, ZEROS, 2, 2, 4>(g, sms, st);
        return rt == 1 ? launch_tile<F16, NG, ZEROS, 4, 1, 4>(g, sms, st) : launch_tile<F16, NG, ZEROS, 4, 2, 4>(g, sms, st);
    }
#endif
    if (g.M <= 8) return launch_tile<F16, NG, ZEROS, 1, 2, 4>(g, sms, st);
    if (g.M <= 16) return launch_tile<F16, NG, ZEROS, 2, 2, 4>(g, sms, st);
    return launch_tile<F16, NG, ZEROS, 4, 2, 4>(g, sms, st);
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
    g.status = status_device_ptr();
    if (sms <= 0 || !g.status) return BS_ERR_CUDA;
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
