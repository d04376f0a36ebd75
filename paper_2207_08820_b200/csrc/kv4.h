// Keys and values of 4 bits in pages: the layout that csrc/kv4_*.cu share.
//
// A page holds `page` entries (tokens) of every head; a head's part of it is one piece of page / 16 tiles, a tile 16 entries, so that one copy
// brings as many neighbouring entries of a head as a page has.  D channels, G = D / group groups.  A tile is
//   keys     16 rows of D / 2 bytes.  Entry r has row r ^ (r >> 2 & 1).  A row is four parts of D / 8 bytes; word w of part t holds the codes of channels
//            32 w + 8 t + (0..7), the lowest bits first: part t is what lane t of a quad multiplies (mma.sync), whatever the group.
//   values   16 rows of D / 2 bytes, entry r in row r.  A row is eight parts of D / 16 bytes; nibble i of part g holds channel 8 i + g: part g is
//            what the lanes that own row g of a fragment multiply.  With D = 128 the parts of entries 2, 3, 6, 7, ... change places by
//            4, with the keys' rows the reason why a fragment's loads meet every bank of shared memory once.
//   steps of the keys, then of the values: 16 entries of G words, the step in the lower half and the offset in the upper one, of the cache's type.
#pragma once
#include <atomic>

#include "common.cuh"

namespace bs {

constexpr int KV4_TILE = 16;        // entries
constexpr int MOST_ROWS = 1 << 30;  // entries or tokens of a call: what loops over them step beyond the last one stays within 31 bits

struct Kv4 {
    unsigned char* data;
    int pages, H, D, page, group, G;
    int log_page;
    int tile;                       // bytes of a tile
    long long head, whole;          // bytes of a head's part of a page, of a page
};

inline bool kv4_layout(const bs_kv4_cache& c, Kv4& l)
{
    if (c.pages <= 0 || c.heads <= 0 || c.heads > 65535) return false;
    if (c.D != 64 && c.D != 96 && c.D != 128) return false;
    if (c.group != 32 && c.group != 64 && c.group != c.D) return false;
    if (c.D % c.group != 0 || c.page < KV4_TILE || c.page > 1024 || (c.page & (c.page - 1))) return false;
    l.data = static_cast<unsigned char*>(c.data);
    l.pages = c.pages; l.H = c.heads; l.D = c.D; l.page = c.page; l.group = c.group; l.G = c.D / c.group;
    for (l.log_page = 4; 1 << l.log_page < c.page; ++l.log_page) {}
    l.tile = KV4_TILE * (c.D + 8 * l.G);
    l.head = static_cast<long long>(c.page / KV4_TILE) * l.tile;
    l.whole = l.head * c.heads;
    return true;
}

// Tables of pages: row b lists the pages of sequence b.
struct Kv4Table {
    const int32_t* pages;
    long long pitch;
    int width, B;
};

#ifdef __CUDACC__
// Lets a kernel have more than 48 KB of shared memory, once a device: the call costs the host half a microsecond.
template <auto KERNEL>
inline bool allow_shared(int bytes)
{
    static std::atomic<unsigned long long> done{0};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) { cudaGetLastError(); return false; }
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return true;
    if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) { cudaGetLastError(); return false; }
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}
// Launch of clusters of `ctas` CTAs that may begin while the kernel before it drains.
template <typename... P, typename... A>
inline int launch_clusters(void (*kern)(P...), unsigned ctas, dim3 grid, dim3 block, size_t smem, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...) != cudaSuccess) {
        cudaGetLastError();
        return BS_ERR_CUDA;
    }
    return BS_OK;
}
__device__ __forceinline__ int kv4_key_row(int r) { return r ^ (r >> 2 & 1); }
__device__ __forceinline__ int kv4_value_part(int D, int r, int g) { return D == 128 ? g ^ (r >> 1 & 1) << 2 : g; }
// Entry i's page, -1 where there is none.  The caller has i below width * page.
__device__ __forceinline__ int kv4_page_of(const Kv4& l, const Kv4Table& t, int b, long long i)
{
    const int p = t.pages[b * t.pitch + (i >> l.log_page)];
    return static_cast<unsigned>(p) < static_cast<unsigned>(l.pages) ? p : -1;
}
__device__ __forceinline__ unsigned char* kv4_tile_of(const Kv4& l, int page, int h, int slot)
{
    return l.data + page * l.whole + h * l.head + static_cast<long long>(slot / KV4_TILE) * l.tile;
}
// The sequence that row i of packed ones belongs to: the largest b with starts[b] <= i (0 where there is none).  starts null: a row each.
__device__ __forceinline__ int kv4_sequence_of(const int32_t* starts, int B, int i)
{
    if (!starts) return i;
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (starts[mid] <= i) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
#endif

}  // namespace bs
