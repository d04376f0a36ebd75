// A mixture-of-experts layer on 4-bit weights for a few tokens, in three launches:
//   route   logits = x R^T, the top_k experts of every token, their softmax weights
//   gate    h[slot] = weight * silu(Gate_e x) * (Up_e x) for every slot (token, choice)
//   down    y[token] = sum over its slots of Down_e h[slot]
// Bound by the bytes of the chosen experts' weights: each of their blocks is read once for up to 64 tokens (more tokens are further passes), through
// shared memory, and multiplied with mma.sync (w4_dot.cuh).  Hidden values stay in 32 bits until they are split in two bf16 terms (hi + lo, 16 bits
// of mantissa), which costs the second product twice the MMAs and no bytes of weights; the range of fp16 would not hold them.
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int PASS = 64;                    // tokens of a pass
constexpr int MAX_EXPERTS = 512, MAX_TOP = 32;
constexpr int ROUTE_CTAS = 8, ROUTE_WARPS = 16;     // CTAs of a cluster, a token each in the end; warps split the reduction
constexpr int WARPS = 8, GATE_STAGES = 4, DOWN_STAGES = 6;

struct MoeArgs {
    const void *x, *router;
    long long ldx;
    int T, E, H, I, top_k, renormalise;
    bool x_aligned, router_aligned;
    const unsigned char *gate, *up, *down;
    W4Layout lu, ld;                        // of one expert's gate or up, and down
    void* xa;                               // aligned copy of x, or null where x is
    long long ldxa;
    __nv_bfloat16 *hi, *lo;                 // [T top_k][ldh]
    int ldh;
    int* experts;
    float* weights;
    void* y;
};

template <typename T>
__device__ __forceinline__ uint4 load8(const T* row, int k0, int K, bool aligned)
{
    if (aligned) return load_x(row, k0, K);
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = k0 + i < K ? __ldg(reinterpret_cast<const uint16_t*>(row) + k0 + i) : 0;
    return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
}

// Whole numbers in the order of the doubles, a NaN above all of them (0 is below all).
__device__ __forceinline__ unsigned long long order_key(double v)
{
    if (isnan(v)) return ~0ull;
    const unsigned long long b = static_cast<unsigned long long>(__double_as_longlong(v == 0.0 ? 0.0 : v));
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

// Logits of eight tokens by a cluster: a CTA takes tiles of 16 experts, its warps split the reduction, each MMA's sum of 16 products is added in 64 bits
// (32 bits would decide the order of experts that are nearly equal by the order of the sums).  CTA r then ranks token r.
template <bool F16>
__global__ void __launch_bounds__(ROUTE_WARPS * 32) w4_moe_route_kernel(const __grid_constant__ MoeArgs g)
{
    typedef W4Type<F16> Ty;
    typedef typename Ty::T T;
    __shared__ double part[ROUTE_WARPS][16][8];
    __shared__ double logits[MAX_EXPERTS];
    __shared__ unsigned long long keys[MAX_EXPERTS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = blockIdx.x, m0 = blockIdx.y * 8;
    const T* x = static_cast<const T*>(dependent_begin(g.x));
    const T* router = static_cast<const T*>(g.router);
    const int tiles = (g.E + 15) / 16, steps = (g.H + 31) / 32;
    const int mx = m0 + (lane >> 2);
    // every CTA of the cluster runs before one writes to another's shared memory
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    for (int tile = rank; tile < tiles; tile += ROUTE_CTAS) {
        const int e0 = tile * 16 + (lane >> 2), e1 = e0 + 8;
        double sum[4] = {0, 0, 0, 0};
#pragma unroll 4
        for (int s = warp; s < steps; s += ROUTE_WARPS) {
            const int k0 = s * 32 + 8 * (lane & 3);
            const uint4 none = make_uint4(0, 0, 0, 0);
            const uint4 a = e0 < g.E ? load8(router + static_cast<size_t>(e0) * g.H, k0, g.H, g.router_aligned) : none;
            const uint4 b = e1 < g.E ? load8(router + static_cast<size_t>(e1) * g.H, k0, g.H, g.router_aligned) : none;
            const uint4 v = mx < g.T ? load8(x + mx * g.ldx, k0, g.H, g.x_aligned) : none;
            float c[4] = {0, 0, 0, 0}, d[4] = {0, 0, 0, 0};
            Ty::mma(c, a.x, b.x, a.y, b.y, v.x, v.y);
            Ty::mma(d, a.z, b.z, a.w, b.w, v.z, v.w);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += static_cast<double>(c[i]) + static_cast<double>(d[i]);
        }
        const int r = lane >> 2, n = 2 * (lane & 3);
        part[warp][r][n] = sum[0];
        part[warp][r][n + 1] = sum[1];
        part[warp][r + 8][n] = sum[2];
        part[warp][r + 8][n + 1] = sum[3];
        __syncthreads();
        if (threadIdx.x < 128) {
            const int e = threadIdx.x >> 3, m = threadIdx.x & 7;
            double v = 0;
#pragma unroll
            for (int k = 0; k < ROUTE_WARPS; ++k) v += part[k][e][m];
            if (tile * 16 + e < g.E) {      // to the CTA that ranks this token
                uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(&logits[tile * 16 + e]));
                asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(to) : "r"(m));
                asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(v) : "memory");
            }
        }
        __syncthreads();
    }
    if (g.xa && m0 + rank < g.T) {      // rows of x on 16-byte boundaries for the next kernel
        T* out = static_cast<T*>(g.xa) + (m0 + rank) * g.ldxa;
        for (int k0 = threadIdx.x * 8; k0 < g.H; k0 += ROUTE_WARPS * 32 * 8)
            *reinterpret_cast<uint4*>(out + k0) = load8(x + (m0 + rank) * g.ldx, k0, g.H, false);
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    const int m = m0 + rank;
    if (warp != 0 || m >= g.T) return;
    // the warp picks the best of what is left, top_k times; lane j keeps choice j
    for (int e = lane; e < g.E; e += 32) keys[e] = order_key(logits[e]);
    __syncwarp();
    int expert = 0;
    for (int j = 0; j < g.top_k; ++j) {
        unsigned long long best = 0;
        int at = MAX_EXPERTS;
        for (int e = lane; e < g.E; e += 32)
            if (keys[e] > best) { best = keys[e]; at = e; }
        const unsigned hi = __reduce_max_sync(0xffffffffu, static_cast<unsigned>(best >> 32));
        const unsigned lo = __reduce_max_sync(0xffffffffu, static_cast<unsigned>(best >> 32) == hi ? static_cast<unsigned>(best) : 0u);
        const int e = __reduce_min_sync(0xffffffffu, best == (static_cast<unsigned long long>(hi) << 32 | lo) ? at : MAX_EXPERTS);     // ties: the lowest index
        if (lane == (e & 31)) keys[e] = 0;      // below every value
        if (lane == j) expert = e;
        __syncwarp();
    }
    const double most = logits[__shfl_sync(0xffffffffu, expert, 0)];
    const float p = lane < g.top_k ? expf(static_cast<float>(logits[expert] - most)) : 0.f;
    float sum = p;
    if (!g.renormalise) {
        sum = 0.f;
        for (int e = lane; e < g.E; e += 32) sum += expf(static_cast<float>(logits[e] - most));
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane < g.top_k) {
        g.experts[m * g.top_k + lane] = expert;
        g.weights[m * g.top_k + lane] = p / sum;
    }
}

// The chosen experts of a pass of 64 tokens and their slots, made by every CTA for itself (at most 2048 slots).
struct Chosen {
    int count[MAX_EXPERTS];             // slots of an expert, then where its next one goes
    int active[MAX_EXPERTS];            // experts that have slots, ascending
    int first[MAX_EXPERTS + 1];         // where the slots of active expert i begin
    int n;
    uint16_t slot[PASS * MAX_TOP];      // slot - first slot of the pass
};

__device__ __forceinline__ void find_chosen(const MoeArgs& g, Chosen& c, int t0, int threads)
{
    const int slots = (g.T - t0 < PASS ? g.T - t0 : PASS) * g.top_k;
    const int* experts = g.experts + static_cast<size_t>(t0) * g.top_k;
    for (int e = threadIdx.x; e < g.E; e += threads) c.count[e] = 0;
    __syncthreads();
    for (int s = threadIdx.x; s < slots; s += threads) atomicAdd(&c.count[experts[s]], 1);
    __syncthreads();
    if (threadIdx.x < 32) {
        int n = 0, at = 0;
        for (int base = 0; base < g.E; base += 32) {
            const int e = base + threadIdx.x, k = e < g.E ? c.count[e] : 0;
            const unsigned has = __ballot_sync(0xffffffffu, k > 0);
            int before = k;             // slots of this and the lower lanes
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, before, d);
                if (static_cast<int>(threadIdx.x) >= d) before += v;
            }
            if (k > 0) {
                const int i = n + __popc(has & ((1u << threadIdx.x) - 1));
                c.active[i] = e;
                c.first[i] = c.count[e] = at + before - k;
            }
            n += __popc(has);
            at += __shfl_sync(0xffffffffu, before, 31);
        }
        if (threadIdx.x == 0) { c.n = n; c.first[n] = at; }
    }
    __syncthreads();
    // the order of an expert's slots is not fixed and does not matter: a slot's results come from its own column
    for (int s = threadIdx.x; s < slots; s += threads) c.slot[atomicAdd(&c.count[experts[s]], 1)] = static_cast<uint16_t>(s);
    __syncthreads();
}

// h = weight * silu(gate) * up of 16 rows of an expert for 16 of its slots at a time; the warps take the blocks of the reduction in turn and copy the
// blocks of the CTA's next items ahead.
template <bool F16, int NG, bool ZEROS>
__global__ void __launch_bounds__(WARPS * 32, 2) w4_moe_gate_kernel(const __grid_constant__ MoeArgs g)
{
    typedef typename W4Type<F16>::T T;
    typedef W4Stage<NG, ZEROS> Stage;
    constexpr int NT = 2, STAGES = GATE_STAGES;
    extern __shared__ __align__(16) unsigned char ring[];      // [WARPS][STAGES][gate, up]
    __shared__ Chosen chosen;
    __shared__ float part[WARPS][2][NT * 8][17];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t0 = blockIdx.y * PASS;
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(ring)) + warp * STAGES * 2 * Stage::BYTES;
    const T* x = static_cast<const T*>(dependent_begin(g.xa ? g.xa : g.x));
    const long long ldx = g.xa ? g.ldxa : g.ldx;
    find_chosen(g, chosen, t0, WARPS * 32);
    const W4Layout& l = g.lu;
    const size_t matrix = l.bytes();
    const int items = chosen.n * l.rbs;
    auto slots = [&](int item) { const int a = item / l.rbs; return chosen.first[a + 1] - chosen.first[a]; };
    // an item whose expert has more than 16 slots is gone through several times
    int citem = blockIdx.x, ccb = warp, cslot = 0, cleft = citem < items ? slots(citem) : 0;
    auto copy = [&] {
        if (citem < items && warp < l.cbs) {
            const int a = citem / l.rbs, rb = citem - a * l.rbs;
            const size_t at = chosen.active[a] * matrix;
            Stage::copy(mine + cslot * 2 * Stage::BYTES, g.gate + at, l, rb, ccb, lane);
            Stage::copy(mine + cslot * 2 * Stage::BYTES + Stage::BYTES, g.up + at, l, rb, ccb, lane);
            ccb += WARPS;
            if (ccb >= l.cbs) {
                ccb = warp;
                cleft -= NT * 8;
                if (cleft <= 0) {
                    citem += gridDim.x;
                    cleft = citem < items ? slots(citem) : 0;
                }
            }
        }
        ring_commit();
        cslot = cslot + 1 == STAGES ? 0 : cslot + 1;
    };
#pragma unroll 1
    for (int s = 0; s < STAGES - 1; ++s) copy();
    int stage = 0;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int a = item / l.rbs, rb = item - a * l.rbs;
        const int beg = chosen.first[a], n = chosen.first[a + 1] - beg;
        for (int s0 = 0; s0 < n; s0 += NT * 8) {
            const T* row[NT];
            float tg[NT][1][4], tu[NT][1][4];
#pragma unroll
            for (int k = 0; k < NT; ++k) {
                const int s = s0 + k * 8 + (lane >> 2);
                row[k] = s < n ? x + (t0 + chosen.slot[beg + s] / g.top_k) * ldx : nullptr;
#pragma unroll
                for (int i = 0; i < 4; ++i) tg[k][0][i] = tu[k][0][i] = 0.f;
            }
            const bool wide = s0 + 8 < n;       // more than eight slots left
            for (int cb = warp; cb < l.cbs; cb += WARPS) {
                uint4 v[1][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[0][j] = row[0] ? load_x(row[0], cb * 128 + 32 * j + 8 * (lane & 3), l.K) : make_uint4(0, 0, 0, 0);
                ring_wait<STAGES - 2>();
                W4Tile<NG, ZEROS> gate, up;
                gate.take(mine + stage * 2 * Stage::BYTES, l, cb, lane);
                up.take(mine + stage * 2 * Stage::BYTES + Stage::BYTES, l, cb, lane);
                stage = stage + 1 == STAGES ? 0 : stage + 1;
                copy();
                w4_block<F16, F16, NG, ZEROS, 1>(gate, v, tg[0]);
                w4_block<F16, F16, NG, ZEROS, 1>(up, v, tu[0]);
                if (wide) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[0][j] = row[1] ? load_x(row[1], cb * 128 + 32 * j + 8 * (lane & 3), l.K) : make_uint4(0, 0, 0, 0);
                    w4_block<F16, F16, NG, ZEROS, 1>(gate, v, tg[1]);
                    w4_block<F16, F16, NG, ZEROS, 1>(up, v, tu[1]);
                }
            }
#pragma unroll
            for (int k = 0; k < NT; ++k) {
                const int m = k * 8 + 2 * (lane & 3), r = lane >> 2;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    part[warp][0][m + (i & 1)][r + 8 * (i >> 1)] = tg[k][0][i];
                    part[warp][1][m + (i & 1)][r + 8 * (i >> 1)] = tu[k][0][i];
                }
            }
            __syncthreads();
            const int m = threadIdx.x >> 4, r = threadIdx.x & 15, i = rb * 16 + r;
            if (s0 + m < n && i < g.I) {
                float gate = 0.f, up = 0.f;
#pragma unroll
                for (int k = 0; k < WARPS; ++k) {
                    gate += part[k][0][m][r];
                    up += part[k][1][m][r];
                }
                const size_t slot = static_cast<size_t>(t0) * g.top_k + chosen.slot[beg + s0 + m];
                const float h = gate / (1.f + expf(-gate)) * up * g.weights[slot];
                const __nv_bfloat16 hi = __float2bfloat16_rn(h);
                g.hi[slot * g.ldh + i] = hi;
                // an infinite or NaN value has no remainder
                g.lo[slot * g.ldh + i] = isfinite(__bfloat162float(hi)) ? __float2bfloat16_rn(h - __bfloat162float(hi)) : __float2bfloat16_rn(0.f);
            }
            __syncthreads();
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// y of 16 columns for the tokens of a pass: the warps share the blocks of all chosen experts, one run of them each, and add up per token in
// shared memory of their own.
template <bool F16, int NG, bool ZEROS>
__global__ void __launch_bounds__(WARPS * 32, 2) w4_moe_down_kernel(const __grid_constant__ MoeArgs g)
{
    typedef typename W4Type<F16>::T T;
    typedef W4Stage<NG, ZEROS> Stage;
    constexpr int STAGES = DOWN_STAGES;
    extern __shared__ __align__(16) unsigned char ring[];      // [WARPS][STAGES] stages, then sums [WARPS][16][pitch]
    __shared__ Chosen chosen;
    float* sums = reinterpret_cast<float*>(ring + WARPS * STAGES * Stage::BYTES);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t0 = blockIdx.y * PASS, rb = blockIdx.x;
    const int tokens = g.T - t0 < PASS ? g.T - t0 : PASS, pitch = tokens + 1;
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(ring)) + warp * STAGES * Stage::BYTES;
    const unsigned char* down = dependent_begin(g.down);
    find_chosen(g, chosen, t0, WARPS * 32);
    const W4Layout& l = g.ld;
    const size_t matrix = l.bytes();
    float* own = sums + warp * 16 * pitch;
    for (int i = lane; i < 16 * pitch; i += 32) own[i] = 0.f;
    __syncwarp();
    const int blocks = chosen.n * l.cbs, beg = static_cast<int>(static_cast<long long>(blocks) * warp / WARPS),
              end = static_cast<int>(static_cast<long long>(blocks) * (warp + 1) / WARPS);
    int cb = beg, ca = beg / l.cbs, cc = beg - ca * l.cbs, cslot = 0;
    auto copy = [&] {
        if (cb < end) {
            Stage::copy(mine + cslot * Stage::BYTES, down + chosen.active[ca] * matrix, l, rb, cc, lane);
            ++cb;
            if (++cc == l.cbs) { cc = 0; ++ca; }
        }
        ring_commit();
        cslot = cslot + 1 == STAGES ? 0 : cslot + 1;
    };
#pragma unroll 1
    for (int s = 0; s < STAGES - 1; ++s) copy();
    int stage = 0, a = beg / l.cbs, c = beg - a * l.cbs;
    for (int b = beg; b < end; ++b) {
        const int first = chosen.first[a], n = chosen.first[a + 1] - first;
        ring_wait<STAGES - 2>();
        W4Tile<NG, ZEROS> tile;
        tile.take(mine + stage * Stage::BYTES, l, c, lane);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        copy();
        for (int s0 = 0; s0 < n; s0 += 8) {
            const int k = s0 + (lane >> 2);
            const size_t slot = static_cast<size_t>(t0) * g.top_k + (k < n ? chosen.slot[first + k] : 0);
            float tot[1][4] = {{0, 0, 0, 0}};
            uint4 hi[1][4], lo[1][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k0 = c * 128 + 32 * j + 8 * (lane & 3);
                hi[0][j] = k < n ? load_x(g.hi + slot * g.ldh, k0, l.K) : make_uint4(0, 0, 0, 0);
                lo[0][j] = k < n ? load_x(g.lo + slot * g.ldh, k0, l.K) : make_uint4(0, 0, 0, 0);
            }
            w4_block<false, F16, NG, ZEROS, 1>(tile, hi, tot);
            w4_block<false, F16, NG, ZEROS, 1>(tile, lo, tot);
#pragma unroll
            for (int i = 0; i < 4; ++i) {       // lanes own different (row, slot): an expert has a token once
                const int q = s0 + 2 * (lane & 3) + (i & 1);
                if (q < n) own[((lane >> 2) + 8 * (i >> 1)) * pitch + chosen.slot[first + q] / g.top_k] += tot[0][i];
            }
        }
        if (++c == l.cbs) { c = 0; ++a; }
        __syncwarp();       // another expert's slots meet the same tokens from other lanes
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * tokens; i += WARPS * 32) {
        const int m = i >> 4, r = i & 15, o = rb * 16 + r;
        if (o >= g.H) continue;
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) v += sums[(k * 16 + r) * pitch + m];
        static_cast<T*>(g.y)[static_cast<size_t>(t0 + m) * g.H + o] = W4Type<F16>::round(v);
    }
}

template <typename K>
bool allow_smem(K kernel, size_t bytes)
{
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)) == cudaSuccess) return true;
    cudaGetLastError();
    return false;
}
template <bool F16, int NG, bool ZEROS>
int launch_gate(const MoeArgs& g, int sms, cudaStream_t st)
{
    const long long slots = static_cast<long long>(g.T < PASS ? g.T : PASS) * g.top_k, items = (slots < g.E ? slots : g.E) * g.lu.rbs;
    const size_t smem = static_cast<size_t>(WARPS) * GATE_STAGES * 2 * W4Stage<NG, ZEROS>::BYTES;
    if (!allow_smem(w4_moe_gate_kernel<F16, NG, ZEROS>, smem)) return BS_ERR_CUDA;
    return launch_dependent(w4_moe_gate_kernel<F16, NG, ZEROS>, dim3(static_cast<unsigned>(items < 2 * sms ? items : 2 * sms), ceil_div(g.T, PASS)),
                            dim3(WARPS * 32), smem, st, g);
}
template <bool F16, int NG, bool ZEROS>
int launch_down(const MoeArgs& g, cudaStream_t st)
{
    const int tokens = g.T < PASS ? g.T : PASS;
    const size_t smem = static_cast<size_t>(WARPS) * (DOWN_STAGES * W4Stage<NG, ZEROS>::BYTES + sizeof(float) * 16 * (tokens + 1));
    if (!allow_smem(w4_moe_down_kernel<F16, NG, ZEROS>, smem)) return BS_ERR_CUDA;
    return launch_dependent(w4_moe_down_kernel<F16, NG, ZEROS>, dim3(g.ld.rbs, ceil_div(g.T, PASS)), dim3(WARPS * 32), smem, st, g);
}
template <bool F16>
int launch_moe(const MoeArgs& g, int sms, cudaStream_t st)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ROUTE_CTAS, ceil_div(g.T, 8));
    cfg.blockDim = dim3(ROUTE_WARPS * 32);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ROUTE_CTAS;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, w4_moe_route_kernel<F16>, g) != cudaSuccess) {
        cudaGetLastError();
        return BS_ERR_CUDA;
    }
    int rc;
    const int nu = g.lu.group == 32 ? 4 : g.lu.group == 64 ? 2 : 1, nd = g.ld.group == 32 ? 4 : g.ld.group == 64 ? 2 : 1;
    if (g.lu.zeros) rc = nu == 4 ? launch_gate<F16, 4, true>(g, sms, st) : nu == 2 ? launch_gate<F16, 2, true>(g, sms, st) : launch_gate<F16, 1, true>(g, sms, st);
    else rc = nu == 4 ? launch_gate<F16, 4, false>(g, sms, st) : nu == 2 ? launch_gate<F16, 2, false>(g, sms, st) : launch_gate<F16, 1, false>(g, sms, st);
    if (rc != BS_OK) return rc;
    if (g.ld.zeros) return nd == 4 ? launch_down<F16, 4, true>(g, st) : nd == 2 ? launch_down<F16, 2, true>(g, st) : launch_down<F16, 1, true>(g, st);
    return nd == 4 ? launch_down<F16, 4, false>(g, st) : nd == 2 ? launch_down<F16, 2, false>(g, st) : launch_down<F16, 1, false>(g, st);
}

size_t hidden_bytes(int T, int top_k, int I) { return static_cast<size_t>(T) * top_k * ((static_cast<size_t>(I) + 7) / 8 * 8) * 2; }
size_t aligned_bytes(int T, int H, long long ldx) { return T == 1 || ldx % 8 == 0 ? 0 : static_cast<size_t>(T) * ((static_cast<size_t>(H) + 7) / 8 * 8) * 2; }

}  // namespace
}  // namespace bs

extern "C" size_t bs_w4_moe_workspace_bytes(int T, int top_k, int H, int I, long long ldx)
{
    if (T <= 0 || top_k <= 0 || H <= 0 || I <= 0) return 0;
    return 2 * bs::hidden_bytes(T, top_k, I) + bs::aligned_bytes(T, H, ldx);
}

extern "C" int bs_w4_moe(const void* x, long long ldx, int T, const void* router, int E, int H, int I, const void* gate, const void* up, int group_up,
                         int zeros_up, const void* down, int group_down, int zeros_down, bs_float_t type, int top_k, int renormalise, void* y,
                         int32_t* experts, float* weights, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace bs;
    MoeArgs g{};
    if (!x || !router || !gate || !up || !down || !y || !experts || !weights || T < 0 || E <= 0 || H <= 0 || I <= 0 || ldx < H || top_k <= 0 ||
        top_k > E || group_up <= 0 || group_down <= 0 || (type != BS_F16 && type != BS_BF16))
        return BS_ERR_INVALID_ARG;
    if (E > MAX_EXPERTS || top_k > MAX_TOP || T > W4_MAX_DIM / PASS || !w4_layout(I, H, group_up, zeros_up, g.lu) || !w4_layout(H, I, group_down, zeros_down, g.ld))
        return BS_ERR_UNSUPPORTED;
    if (!aligned16(x) || !aligned16(router) || !aligned16(gate) || !aligned16(up) || !aligned16(down) || !aligned16(y) || !aligned16(experts) ||
        !aligned16(weights) || !aligned16(workspace))
        return BS_ERR_ALIGNMENT;
    if (T == 0) return BS_OK;
    if (!workspace || workspace_bytes < bs_w4_moe_workspace_bytes(T, top_k, H, I, ldx)) return BS_ERR_INVALID_ARG;
    g.x = x; g.router = router; g.ldx = ldx; g.T = T; g.E = E; g.H = H; g.I = I; g.top_k = top_k; g.renormalise = renormalise != 0;
    g.x_aligned = aligned_bytes(T, H, ldx) == 0;
    g.router_aligned = E == 1 || H % 8 == 0;
    g.gate = static_cast<const unsigned char*>(gate); g.up = static_cast<const unsigned char*>(up); g.down = static_cast<const unsigned char*>(down);
    g.ldh = (I + 7) & ~7;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    g.hi = reinterpret_cast<__nv_bfloat16*>(ws);
    g.lo = reinterpret_cast<__nv_bfloat16*>(ws + hidden_bytes(T, top_k, I));
    if (!g.x_aligned) {
        g.xa = ws + 2 * hidden_bytes(T, top_k, I);
        g.ldxa = (H + 7) & ~7;
    }
    g.experts = experts; g.weights = weights; g.y = y;
    const int sms = device_sm_count();
    if (sms <= 0) return BS_ERR_CUDA;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return type == BS_F16 ? launch_moe<true>(g, sms, st) : launch_moe<false>(g, sms, st);
}
