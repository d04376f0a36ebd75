// A mixture-of-experts layer on 4-bit weights for a few tokens, in four launches:
//   route   logits = x R^T, the top_k experts of every token, their softmax weights
//   gate    h[slot] = weight * silu(Gate_e x) * (Up_e x) for every slot (token, choice)
//   down    z[slot] = Down_e h[slot]
//   sum     y[token] = sum over its slots of z[slot]
// Each block of the chosen experts' weights comes from HBM once for up to 64 tokens (more tokens are further passes), through shared memory, and is multiplied
// with mma.sync (w4_dot.cuh).  What bounds it: for one token the four launches (12 us with next to no weights; 64 experts of 2048 x 1024, 8 chosen: 24.6 us, of
// which their bytes take 4), with more the expansion of the codes, which fills half of the issue slots, and x, hidden values and sums, which 17 warps an SM wait for
// (64 tokens, 128 experts of 2048 x 768, 126 of them chosen: 121 us, 2.5 TB/s; 8 tokens, 2 of 16 experts of 4096 x 8192, alone: 137 us with 8 of them chosen, 160
// with 10, 184 with 12, 3.0 to 3.4 TB/s).  Hidden values stay in 32 bits until they are split in two bf16 terms (hi + lo, 16 bits of mantissa and the sign
// between them), which costs the second product twice the MMAs and no bytes of weights; the range of fp16 would not hold them.  All 24 bits, as three terms split in the
// second product from the 32-bit values, took 139 us in place of 121; the error against 64 bits, which the rounding of y makes, is that of float32 hidden
// values to five digits in bf16, four in fp16.
#include "w4_dot.cuh"

namespace bs {
namespace {

constexpr int PASS = 64;                    // tokens of a pass
constexpr int MAX_EXPERTS = 512, MAX_TOP = 32;
constexpr int ROUTE_CTAS = 8, ROUTE_WARPS = 16;     // CTAs of a cluster, a token each in the end; warps split the reduction
constexpr int WARPS = 8, GATE_STAGES = 4, DOWN_STAGES = 4;

struct MoeArgs {
    const void *x, *router;
    long long ldx;
    int T, E, H, I, top_k, renormalise;
    bool x_aligned, router_aligned;
    const unsigned char *gate, *up, *down;
    W4Layout lu, ld;                        // of one expert's gate or up, and down
    CUtensorMap tg, tu, td;                 // their blocks, in boxes of a CTA's teams
    int down_split, down_ctas;              // of the second product: warps of a team, CTAs
    void* xa;                               // aligned copy of x, or null where x is
    long long ldxa;
    __nv_bfloat16 *hi, *lo;                 // [T top_k][ldh]
    float* z;                               // [T top_k][ldz]
    int ldh, ldz;
    int* status;                            // device status word
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

// Whole numbers in the order of the doubles, a NaN above all of them.
__device__ __forceinline__ unsigned long long order_key(double v)
{
    if (isnan(v)) return ~0ull;
    const unsigned long long b = static_cast<unsigned long long>(__double_as_longlong(v == 0.0 ? 0.0 : v));
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

// An MMA's sum of 16 products is at most this far off, of their magnitudes' sum: it holds 24 bits of the largest one's place, so that 15 products lose less than
// 2^-23 of it each and the sum as much again; a sixteenth more for the sum of the magnitudes, which is in 32 bits itself.
constexpr float SUM_CUT = 1.0625f / (1 << 19);

// The logits of the experts that `open` names, from products that are exact in 64 bits and summed there: warps share the columns, `parts` [OPEN][ROUTE_WARPS] holds
// their sums.  All threads.  Not inlined: few tokens need it, and its instructions would be in the others' way.
constexpr int OPEN = 128;       // experts at a time
template <bool F16>
__device__ __noinline__ void exact_logits(const MoeArgs& g, const typename W4Type<F16>::T* x, const typename W4Type<F16>::T* router, const unsigned char* open, double* parts, double* logits)
{
    typedef W4Type<F16> Ty;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int first = 0; first < g.E; first += OPEN) {
        for (int at = 0; at < OPEN; at += 32) {
            const int e = first + at + lane;
            for (unsigned left = __ballot_sync(0xffffffffu, e < g.E && open[e]); left; left &= left - 1) {
                const int i = at + __ffs(left) - 1;
                const auto* row = router + static_cast<size_t>(first + i) * g.H;
                double s[2] = {0, 0};
                for (int k0 = threadIdx.x * 8; k0 < g.H; k0 += ROUTE_WARPS * 32 * 8) {
                    const uint4 v = load8(x, k0, g.H, g.x_aligned), w = load8(row, k0, g.H, g.router_aligned);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[0] = fma(static_cast<double>(Ty::lo(word_of(v, j))), static_cast<double>(Ty::lo(word_of(w, j))), s[0]);
                        s[1] = fma(static_cast<double>(Ty::hi(word_of(v, j))), static_cast<double>(Ty::hi(word_of(w, j))), s[1]);
                    }
                }
                s[0] += s[1];
#pragma unroll
                for (int d = 16; d; d >>= 1) s[0] += __shfl_xor_sync(0xffffffffu, s[0], d);
                if (lane == 0) parts[i * ROUTE_WARPS + warp] = s[0];
            }
        }
        __syncthreads();
        const int i = threadIdx.x;
        if (i < OPEN && first + i < g.E && open[first + i]) {
            double s = 0;
            for (int k = 0; k < ROUTE_WARPS; ++k) s += parts[i * ROUTE_WARPS + k];
            logits[first + i] = s;
        }
        __syncthreads();
    }
}

// Logits of eight tokens by a cluster: a CTA takes tiles of 16 experts, its warps split the reduction, each MMA's sum of 16 products is added in 64 bits, and
// the products' magnitudes by MMAs beside them.  CTA r then ranks token r.  What an MMA cuts off can exceed what two logits differ by: experts that may change
// places with a chosen one get their products summed in 64 bits, one by one, and are ranked again (one token in a hundred, 8 of 128 experts of normal weights
// and 2048 columns).  The check takes 0.6 us (1 token, 8 of 64 experts of 2048 x 1024: 24.6 in place of 24.1), and with it 64 tokens of 128 experts of 2048 x 768 take
// 121 in place of 119, as nearly every other call has such a token.
template <bool F16>
__global__ void __launch_bounds__(ROUTE_WARPS * 32) w4_moe_route_kernel(const __grid_constant__ MoeArgs g)
{
    typedef W4Type<F16> Ty;
    typedef typename Ty::T T;
    __shared__ double part[ROUTE_WARPS][16][8];
    __shared__ double logits[MAX_EXPERTS];
    __shared__ float sizes[ROUTE_WARPS][16][8], cut[MAX_EXPERTS];       // cut: how far a logit may be off
    __shared__ unsigned long long keys[MAX_EXPERTS];
    __shared__ unsigned char open[MAX_EXPERTS];
    __shared__ int choice[MAX_TOP];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = blockIdx.x, m0 = blockIdx.y * 8;
    const int tiles = (g.E + 15) / 16, steps = (g.H + 31) / 32;
    // the router's rows start for L2 while the kernel in front drains
    if (blockIdx.y == 0 && threadIdx.x < 16)
        for (int e = rank * 16 + threadIdx.x; e < g.E; e += ROUTE_CTAS * 16) {
            const unsigned long long row = (reinterpret_cast<unsigned long long>(g.router) + static_cast<size_t>(e) * g.H * 2) & ~15ull;
            if (g.H >= 8) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row), "r"(g.H / 8 * 16) : "memory");
        }
    const T* x = static_cast<const T*>(dependent_begin(g.x));
    const T* router = behind_wait<T>(g.router);
    const int mx = m0 + (lane >> 2);
    // every CTA of the cluster runs before one writes to another's shared memory
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    for (int tile = rank; tile < tiles; tile += ROUTE_CTAS) {
        const int e0 = tile * 16 + (lane >> 2), e1 = e0 + 8;
        double sum[4] = {0, 0, 0, 0};
        float size[4] = {0, 0, 0, 0};
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
            const uint32_t m = 0x7fff7fffu;
            Ty::mma(size, a.x & m, b.x & m, a.y & m, b.y & m, v.x & m, v.y & m);
            Ty::mma(size, a.z & m, b.z & m, a.w & m, b.w & m, v.z & m, v.w & m);
        }
        const int r = lane >> 2, n = 2 * (lane & 3);
        part[warp][r][n] = sum[0];
        part[warp][r][n + 1] = sum[1];
        part[warp][r + 8][n] = sum[2];
        part[warp][r + 8][n + 1] = sum[3];
        sizes[warp][r][n] = size[0];
        sizes[warp][r][n + 1] = size[1];
        sizes[warp][r + 8][n] = size[2];
        sizes[warp][r + 8][n + 1] = size[3];
        __syncthreads();
        if (threadIdx.x < 128) {
            const int e = threadIdx.x >> 3, m = threadIdx.x & 7;
            double v = 0;
            float far = 0;
#pragma unroll
            for (int k = 0; k < ROUTE_WARPS; ++k) {
                v += part[k][e][m];
                far += sizes[k][e][m];
            }
            if (tile * 16 + e < g.E) {      // to the CTA that ranks this token
                uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(&logits[tile * 16 + e])), at = static_cast<uint32_t>(__cvta_generic_to_shared(&cut[tile * 16 + e]));
                asm volatile("mapa.shared::cluster.u32 %0, %0, %2;\n\tmapa.shared::cluster.u32 %1, %1, %2;" : "+r"(to), "+r"(at) : "r"(m));
                asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(v) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(far * SUM_CUT) : "memory");
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
    if (m >= g.T) return;
    // an expert's place is the number of experts before it: larger logits, and equal ones of lower index.  `share` neighbouring threads count for one.
    int share = 32;
    while (share > 1 && share * g.E > ROUTE_WARPS * 32) share /= 2;
    const int e = threadIdx.x / share, turn = threadIdx.x % share;
    for (bool again = false;; again = true) {
        for (int i = threadIdx.x; i < g.E; i += ROUTE_WARPS * 32) {
            keys[i] = order_key(logits[i]);
            open[i] = 0;
        }
        __syncthreads();
        int place = 0;
        if (e < g.E) {
            const unsigned long long key = keys[e];
            for (int k = turn; k < g.E; k += share) place += keys[k] > key || (keys[k] == key && k < e);
        }
        for (int d = 1; d < share; d <<= 1) place += __shfl_xor_sync(0xffffffffu, place, d);
        if (e < g.E && turn == 0 && place < g.top_k) choice[place] = e;
        __syncthreads();
        if (again) break;
        bool near = false;
        if (e < g.E) {
            const double own = logits[e];
            const float far = cut[e];
            for (int c = turn; c < g.top_k; c += share) {
                const int k = choice[c];
                const float both = far + cut[k];        // 0: a token of zeros, whose sums are exact
                if (k != e && both > 0 && fabs(own - logits[k]) <= both) near = open[e] = open[k] = 1;
            }
        }
        if (!__syncthreads_or(near)) break;
        // what is not open keeps its order with all that is: it is farther from every chosen expert than both sums may be off
        static_assert(sizeof(part) == OPEN * ROUTE_WARPS * sizeof(double), "the sums' place");
        exact_logits<F16>(g, x + m * g.ldx, router, open, &part[0][0][0], logits);
    }
    if (warp != 0) return;
    const int expert = lane < g.top_k ? choice[lane] : 0;
    const double most = logits[choice[0]];
    const float p = lane < g.top_k ? expf(static_cast<float>(logits[expert] - most)) : 0.f;
    float sum = p;
    if (!g.renormalise) {
        sum = 0.f;
        for (int k = lane; k < g.E; k += 32) sum += expf(static_cast<float>(logits[k] - most));
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane < g.top_k) {
        g.experts[m * g.top_k + lane] = expert;
        g.weights[m * g.top_k + lane] = p / sum;
    }
}

// The work of a pass of 64 tokens: jobs of an expert and up to eight of its slots, made by every CTA for itself (at most 2048 slots).  An expert of more slots
// has several jobs, which read its weights again, from L2: jobs of 16 slots (two tiles of x, twice the registers) took 105 us where these take 100,
// with 16 slots an expert (64 tokens, 2 of 8 experts, 2048 x 4096), and 77 to 68 with eight.
constexpr int J = 8, MOST_JOBS = MAX_EXPERTS + PASS * MAX_TOP / J;
struct Jobs {
    unsigned tokens[2][MAX_EXPERTS];    // which tokens chose an expert, a bit each
    uint16_t begin[MAX_EXPERTS];        // where an expert's slots begin
    uint16_t expert[MOST_JOBS];
    uint16_t first[MOST_JOBS + 1];      // where the slots of a job begin
    uint16_t slot[PASS * MAX_TOP];      // slot - first slot of the pass; by expert, then by token, in every CTA alike
    uint8_t token[PASS * MAX_TOP];      // its token - first token of the pass
    int n;
};

__device__ __forceinline__ void find_jobs(const MoeArgs& g, Jobs& c, int t0, int threads)
{
    const int slots = (g.T - t0 < PASS ? g.T - t0 : PASS) * g.top_k;
    const int* experts = g.experts + static_cast<size_t>(t0) * g.top_k;
    if (slots == g.top_k) {     // one token: its experts are all different, a job each; a search of 1.2 us less in either product
        for (int s = threadIdx.x; s < slots; s += threads) {
            c.expert[s] = static_cast<uint16_t>(experts[s]);
            c.first[s] = c.slot[s] = static_cast<uint16_t>(s);
            c.token[s] = 0;
        }
        if (threadIdx.x == 0) { c.n = slots; c.first[slots] = static_cast<uint16_t>(slots); }
        __syncthreads();
        return;
    }
    for (int e = threadIdx.x; e < g.E; e += threads) c.tokens[0][e] = c.tokens[1][e] = 0;
    __syncthreads();
    for (int s = threadIdx.x; s < slots; s += threads) {
        const int t = s / g.top_k;
        atomicOr(&c.tokens[t >> 5][experts[s]], 1u << (t & 31));
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        int jobs = 0, at = 0;
        for (int base = 0; base < g.E; base += 32) {
            const int e = base + threadIdx.x, k = e < g.E ? __popc(c.tokens[0][e]) + __popc(c.tokens[1][e]) : 0, own = (k + J - 1) / J;
            int before = own << 16 | k;             // jobs and slots of this and the lower lanes
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, before, d);
                if (static_cast<int>(threadIdx.x) >= d) before += v;
            }
            const int j0 = jobs + (before >> 16) - own, s0 = at + (before & 0xffff) - k;
            if (e < g.E) c.begin[e] = static_cast<uint16_t>(s0);
            for (int j = 0; j < own; ++j) {
                c.expert[j0 + j] = static_cast<uint16_t>(e);
                c.first[j0 + j] = static_cast<uint16_t>(s0 + j * J);
            }
            const int all = __shfl_sync(0xffffffffu, before, 31);
            jobs += all >> 16;
            at += all & 0xffff;
        }
        if (threadIdx.x == 0) { c.n = jobs; c.first[jobs] = static_cast<uint16_t>(at); }
    }
    __syncthreads();
    for (int s = threadIdx.x; s < slots; s += threads) {
        const int t = s / g.top_k, e = experts[s];
        const unsigned lower = (1u << (t & 31)) - 1;
        const int i = c.begin[e] + (t < 32 ? __popc(c.tokens[0][e] & lower) : __popc(c.tokens[0][e]) + __popc(c.tokens[1][e] & lower));
        c.slot[i] = static_cast<uint16_t>(s);
        c.token[i] = static_cast<uint8_t>(t);
    }
    __syncthreads();
}

// h = weight * silu(gate) * up of 16 rows of an expert for the slots of a job.  The warps of a team share the reduction of 16 rows; the last warp copies
// the blocks of the CTA's items ahead, also while the sums of an item are put together.
template <bool F16, int NG, bool ZEROS>
__global__ void __launch_bounds__(WARPS * 32 + 32, 2) w4_moe_gate_kernel(const __grid_constant__ MoeArgs g, int split)
{
    typedef typename W4Type<F16>::T T;
    typedef W4TeamRing<NG, ZEROS, 2, WARPS, GATE_STAGES> Ring;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[2 * GATE_STAGES];
    __shared__ Jobs jobs;
    __shared__ float parts[2][WARPS][2][J][17];     // items take turns: one barrier each
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t0 = blockIdx.y * PASS;
    const int team = warp / split, k0 = warp % split, teams = WARPS / split;
    Ring ring(smem, bars, warp, lane);
    const T* x = static_cast<const T*>(dependent_begin(g.xa ? g.xa : g.x));
    const long long ldx = g.xa ? g.ldxa : g.ldx;
    find_jobs(g, jobs, t0, WARPS * 32 + 32);
    const W4Layout& l = g.lu;
    // an item: a job and the rows of all teams
    const int per_job = (l.rbs + teams - 1) / teams, items = jobs.n * per_job, full = l.K / W4_COLS;
    if (warp == WARPS) {
        const CUtensorMap* const maps[2] = {&g.tg, &g.tu};
        if (lane == 0) {
            int filled = 0;
            for (int item = blockIdx.x; item < items; item += gridDim.x) {
                const int job = item / per_job, rb0 = (item - job * per_job) * teams;
                for (int c = 0; c < l.cbs; c += split, ++filled) ring.fill(maps, {rb0, rb0}, c, jobs.expert[job], g.status);
            }
            // what the second product's CTA of this place takes first starts for L2 (one token, 2 of 16 experts of 4096 x 4096: 31.4 in place of 32.2 us)
            const int high = WARPS / g.down_split, per_down = (g.ld.rbs + 2 * high - 1) / (2 * high);
            int left = DOWN_STAGES;
            for (int item = blockIdx.x; item < jobs.n * per_down && left > 0; item += g.down_ctas) {
                const int job = item / per_down, rb0 = (item - job * per_down) * 2 * high;
                for (int c = 0; c < g.ld.cbs && left > 0; c += g.down_split, --left) {
                    Ring::hint(&g.td, rb0, c, jobs.expert[job]);
                    Ring::hint(&g.td, rb0 + high, c, jobs.expert[job]);
                }
            }
            ring.drain(filled, g.status);
        }
        return;
    }
    int turn = 0;
    for (int item = blockIdx.x; item < items; item += gridDim.x, turn ^= 1) {
        float (*part)[2][J][17] = parts[turn];
        const int job = item / per_job, rb = (item - job * per_job) * teams + team, beg = jobs.first[job];
        // a job's slots end where the next one's begin; lanes without a slot compute the last one's again
        const int n = jobs.first[job + 1] - beg;
        const T* row = x + (t0 + jobs.token[beg + min(lane >> 2, n - 1)]) * ldx + 8 * (lane & 3);
        float tot[2][1][4] = {};
        // teams without rows multiply what the stages hold, and drop it
        for (int c = k0; c < l.cbs + k0; c += split) {
            uint4 v[4];
            if (c < l.cbs) load_block_x(v, row, c, l.K, c < full, lane);
            ring.landed(g.status);
            if (c < l.cbs) {
                W4Tile<NG, ZEROS> w[2];
                ring.take(w);
                w4_blocks<F16, F16, 1>(w, [&](int, int j, int) { return v[j]; }, tot);
            }
            ring.release(lane);
            ring.next();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = 2 * (lane & 3) + (i & 1), r = (lane >> 2) + 8 * (i >> 1);
            part[warp][0][m][r] = tot[0][0][i];
            part[warp][1][m][r] = tot[1][0][i];
        }
        asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 * split) : "memory");
        for (int q = k0 * 32 + lane; q < J * 16; q += 32 * split) {
            const int m = q >> 4, r = q & 15, i = rb * 16 + r;
            if (m >= n || i >= g.I) continue;
            float gate = 0.f, up = 0.f;
            for (int k = 0; k < split; ++k) {
                gate += part[team * split + k][0][m][r];
                up += part[team * split + k][1][m][r];
            }
            gate *= W4Type<F16>::PART;
            up *= W4Type<F16>::PART;
            const size_t slot = static_cast<size_t>(t0) * g.top_k + jobs.slot[beg + m];
            const float h = gate / (1.f + expf(-gate)) * up * g.weights[slot];
            const __nv_bfloat16 hi = __float2bfloat16_rn(h);
            g.hi[slot * g.ldh + i] = hi;
            // an infinite or NaN value has no remainder
            g.lo[slot * g.ldh + i] = isfinite(__bfloat162float(hi)) ? __float2bfloat16_rn(h - __bfloat162float(hi)) : __float2bfloat16_rn(0.f);
        }
    }
}

// z = Down_e h of 32 rows of an expert for the slots of a job, items and teams as above.  32 rows a warp, because the hidden values of eight slots are four
// times the weights' bytes that they meet in 16.  (With the tokens' sums kept in the CTA instead, job after job, a job's few blocks waited for
// barriers: 95 us where this and the sums behind it took 64, 64 tokens of 128 experts.)
template <bool F16, int NG, bool ZEROS>
__global__ void __launch_bounds__(WARPS * 32 + 32, 2) w4_moe_down_kernel(const __grid_constant__ MoeArgs g, int split)
{
    typedef W4TeamRing<NG, ZEROS, 2, WARPS, DOWN_STAGES> Ring;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[2 * DOWN_STAGES];
    __shared__ Jobs jobs;
    __shared__ float parts[2][WARPS][J][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t0 = blockIdx.y * PASS;
    const int team = warp / split, k0 = warp % split, teams = WARPS / split;
    Ring ring(smem, bars, warp, lane);
    dependent_begin(g.down);
    const __nv_bfloat16* hidden = behind_wait<__nv_bfloat16>(g.hi);
    find_jobs(g, jobs, t0, WARPS * 32 + 32);
    const W4Layout& l = g.ld;
    const int per_job = (l.rbs + 2 * teams - 1) / (2 * teams), items = jobs.n * per_job, full = l.K / W4_COLS;
    if (warp == WARPS) {
        const CUtensorMap* const maps[2] = {&g.td, &g.td};
        if (lane == 0) {
            int filled = 0;
            for (int item = blockIdx.x; item < items; item += gridDim.x) {
                const int job = item / per_job, rb0 = (item - job * per_job) * 2 * teams;
                for (int c = 0; c < l.cbs; c += split, ++filled) ring.fill(maps, {rb0, rb0 + teams}, c, jobs.expert[job], g.status);
            }
            ring.drain(filled, g.status);
        }
        return;
    }
    const long long lo = g.lo - g.hi;
    int turn = 0;
    for (int item = blockIdx.x; item < items; item += gridDim.x, turn ^= 1) {
        float (*part)[J][33] = parts[turn];
        const int job = item / per_job, rb = (item - job * per_job) * 2 * teams + team, beg = jobs.first[job], n = jobs.first[job + 1] - beg;
        const size_t slot0 = static_cast<size_t>(t0) * g.top_k;
        const __nv_bfloat16* row = hidden + (slot0 + jobs.slot[beg + min(lane >> 2, n - 1)]) * g.ldh + 8 * (lane & 3);
        float tot[2][1][4] = {};
        // teams without rows multiply what the stages hold, and drop it
        for (int c = k0; c < l.cbs + k0; c += split) {
            uint4 v[2][4];          // both terms on their way while the weights are waited for
            if (c < l.cbs) {
                load_block_x(v[0], row, c, l.K, c < full, lane);
                load_block_x(v[1], row + lo, c, l.K, c < full, lane);
            }
            ring.landed(g.status);
            if (c < l.cbs) {
                W4Tile<NG, ZEROS> w[2];
                ring.take(w);
                w4_blocks<false, F16, 2>(w, [&](int, int j, int t) { return v[t][j]; }, tot);
            }
            ring.release(lane);
            ring.next();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = 2 * (lane & 3) + (i & 1), r = (lane >> 2) + 8 * (i >> 1);
            part[warp][m][r] = tot[0][0][i];
            part[warp][m][r + 16] = tot[1][0][i];
        }
        asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 * split) : "memory");
        for (int q = k0 * 32 + lane; q < n * 32; q += 32 * split) {
            const int m = q >> 5, r = q & 31, o = (rb + (r >> 4) * teams) * 16 + (r & 15);      // two blocks of rows, `teams` apart
            if (o >= g.H) continue;
            float v = 0.f;
            for (int k = 0; k < split; ++k) v += part[team * split + k][m][r];
            g.z[(slot0 + jobs.slot[beg + m]) * g.ldz + o] = v * W4Type<false>::PART;
        }
    }
}

// y[token] = the sum of its slots' z, in the order of the choices.  A thread: four columns.
template <bool F16>
__global__ void __launch_bounds__(256) w4_moe_sum_kernel(const __grid_constant__ MoeArgs g)
{
    typedef typename W4Type<F16>::T T;
    const float* z = dependent_begin(g.z);
    const int quads = g.ldz / 4, step = gridDim.x * blockDim.x;
    for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < static_cast<long long>(g.T) * quads; i += step) {
        const int t = static_cast<int>(i / quads), h = static_cast<int>(i - static_cast<long long>(t) * quads) * 4;
        const float* p = z + static_cast<size_t>(t) * g.top_k * g.ldz + h;
        float4 v = *reinterpret_cast<const float4*>(p);
#pragma unroll 8
        for (int j = 1; j < g.top_k; ++j) {
            const float4 w = *reinterpret_cast<const float4*>(p + static_cast<size_t>(j) * g.ldz);
            v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
        }
        T* y = static_cast<T*>(g.y) + static_cast<size_t>(t) * g.H + h;
        if (g.H % 4 == 0) {
            *reinterpret_cast<uint2*>(y) = make_uint2(W4Type<F16>::round2(v.x, v.y), W4Type<F16>::round2(v.z, v.w));
        } else {
            const float s[4] = {v.x, v.y, v.z, v.w};
            for (int k = 0; k < 4 && h + k < g.H; ++k) y[k] = W4Type<F16>::round(s[k]);
        }
    }
}

template <typename K>
bool allow_smem(K kernel, size_t bytes)
{
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)) == cudaSuccess) return true;
    cudaGetLastError();
    return false;
}
// Launch of a kernel of clusters that may begin while the one before it drains.
template <typename... P, typename... A>
int launch_clusters(void (*kern)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...) == cudaSuccess) return BS_OK;
    cudaGetLastError();
    return BS_ERR_CUDA;
}
// The most jobs that a pass can have, as find_jobs cuts them: a slot each, or one more than its slots fill for every expert.
int most_jobs(const MoeArgs& g)
{
    const int slots = (g.T < PASS ? g.T : PASS) * g.top_k, cut = g.E + slots / J;
    return slots < cut ? slots : cut;
}
template <bool F16, int NG, bool ZEROS>
int launch_gate(MoeArgs& g, int sms, cudaStream_t st)
{
    const int split = w4_team_width(WARPS, g.lu.cbs);
    const long long items = static_cast<long long>(most_jobs(g)) * ceil_div(g.lu.rbs, WARPS / split);
    constexpr int smem = W4TeamRing<NG, ZEROS, 2, WARPS, GATE_STAGES>::BYTES;
    if (!allow_smem(w4_moe_gate_kernel<F16, NG, ZEROS>, smem) || !w4_encode_blocks(&g.tg, g.gate, g.lu, g.E, split, WARPS / split) ||
        !w4_encode_blocks(&g.tu, g.up, g.lu, g.E, split, WARPS / split))
        return BS_ERR_CUDA;
    return launch_dependent(w4_moe_gate_kernel<F16, NG, ZEROS>, dim3(static_cast<unsigned>(items < 2 * sms ? items : 2 * sms), ceil_div(g.T, PASS)),
                            dim3(WARPS * 32 + 32), smem, st, g, split);
}
template <bool F16, int NG, bool ZEROS>
int launch_down(MoeArgs& g, cudaStream_t st)
{
    constexpr int smem = W4TeamRing<NG, ZEROS, 2, WARPS, DOWN_STAGES>::BYTES;
    if (!allow_smem(w4_moe_down_kernel<F16, NG, ZEROS>, smem)) return BS_ERR_CUDA;
    return launch_dependent(w4_moe_down_kernel<F16, NG, ZEROS>, dim3(static_cast<unsigned>(g.down_ctas), ceil_div(g.T, PASS)), dim3(WARPS * 32 + 32), smem, st, g,
                            g.down_split);
}
template <bool F16>
int launch_experts(MoeArgs& g, int sms, cudaStream_t st)
{
    int rc;
    const int nu = g.lu.group == 32 ? 4 : g.lu.group == 64 ? 2 : 1, nd = g.ld.group == 32 ? 4 : g.ld.group == 64 ? 2 : 1;
    if (g.lu.zeros) rc = nu == 4 ? launch_gate<F16, 4, true>(g, sms, st) : nu == 2 ? launch_gate<F16, 2, true>(g, sms, st) : launch_gate<F16, 1, true>(g, sms, st);
    else rc = nu == 4 ? launch_gate<F16, 4, false>(g, sms, st) : nu == 2 ? launch_gate<F16, 2, false>(g, sms, st) : launch_gate<F16, 1, false>(g, sms, st);
    if (rc != BS_OK) return rc;
    if (g.ld.zeros) return nd == 4 ? launch_down<F16, 4, true>(g, st) : nd == 2 ? launch_down<F16, 2, true>(g, st) : launch_down<F16, 1, true>(g, st);
    return nd == 4 ? launch_down<F16, 4, false>(g, st) : nd == 2 ? launch_down<F16, 2, false>(g, st) : launch_down<F16, 1, false>(g, st);
}
template <bool F16>
int launch_moe(MoeArgs& g, int sms, cudaStream_t st)
{
    int rc = launch_clusters(w4_moe_route_kernel<F16>, dim3(ROUTE_CTAS, ceil_div(g.T, 8)), ROUTE_WARPS * 32, 0, ROUTE_CTAS, st, g);
    if (rc != BS_OK) return rc;
    g.down_split = w4_team_width(WARPS, g.ld.cbs);
    const long long items = static_cast<long long>(most_jobs(g)) * ceil_div(g.ld.rbs, 2 * WARPS / g.down_split);
    g.down_ctas = static_cast<int>(items < 2 * sms ? items : 2 * sms);
    if (!w4_encode_blocks(&g.td, g.down, g.ld, g.E, g.down_split, WARPS / g.down_split)) return BS_ERR_CUDA;
    rc = launch_experts<F16>(g, sms, st);
    if (rc != BS_OK) return rc;
    const long long want = (static_cast<long long>(g.T) * (g.ldz / 4) + 255) / 256, most = 8ll * sms;
    return launch_dependent(w4_moe_sum_kernel<F16>, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(256), 0, st, g);
}

size_t slot_bytes(int T, int top_k, int H) { return static_cast<size_t>(T) * top_k * ((static_cast<size_t>(H) + 3) / 4 * 4) * 4; }
size_t hidden_bytes(int T, int top_k, int I) { return static_cast<size_t>(T) * top_k * ((static_cast<size_t>(I) + 7) / 8 * 8) * 2; }
size_t aligned_bytes(int T, int H, long long ldx) { return T == 1 || ldx % 8 == 0 ? 0 : static_cast<size_t>(T) * ((static_cast<size_t>(H) + 7) / 8 * 8) * 2; }

}  // namespace
}  // namespace bs

extern "C" size_t bs_w4_moe_workspace_bytes(int T, int top_k, int H, int I, long long ldx)
{
    if (T <= 0 || top_k <= 0 || H <= 0 || I <= 0) return 0;
    return bs::slot_bytes(T, top_k, H) + 2 * bs::hidden_bytes(T, top_k, I) + bs::aligned_bytes(T, H, ldx);
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
    g.z = reinterpret_cast<float*>(ws);
    g.ldz = (H + 3) & ~3;
    ws += slot_bytes(T, top_k, H);
    g.hi = reinterpret_cast<__nv_bfloat16*>(ws);
    g.lo = reinterpret_cast<__nv_bfloat16*>(ws + hidden_bytes(T, top_k, I));
    if (!g.x_aligned) {
        g.xa = ws + 2 * hidden_bytes(T, top_k, I);
        g.ldxa = (H + 7) & ~7;
    }
    g.experts = experts; g.weights = weights; g.y = y;
    g.status = status_device_ptr();
    const int sms = device_sm_count();
    if (sms <= 0 || !g.status) return BS_ERR_CUDA;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return type == BS_F16 ? launch_moe<true>(g, sms, st) : launch_moe<false>(g, sms, st);
}
