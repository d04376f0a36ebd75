// Weights of 4 bits with a scale (and zero point) per group of the reduction, laid out for the tensor cores: shared by csrc/w4_*.cu.
//
// A prepared matrix of O rows and K columns is [ceil(O/16)][ceil(K/128)] blocks of 16 rows and 128 columns, each in one piece, which one bulk copy moves:
//   codes  [t 0..3][16 bytes of a row, 16 rows]: word j of the 16 bytes holds the stored codes (0..15) of columns 32 j + 8 t + (0..7): nibble i < 4 is
//          column 2 i, nibble i >= 4 column 2 (i - 4) + 1, so that (word >> 4 i) & 0x000f000f is a pair of neighbouring columns, one in each
//          half.  The 16 bytes are one row's part of what lane t of a quad multiplies (mma.sync), and four of them are a row's 128 columns
//          for the thread that owns the row (tensor memory).  Row r has place (r & 8) | ((r & 7) ^ 2 t): either way of reading meets
//          every bank of shared memory once.
//   steps  [groups in the block: 4, 2 or 1][8 entries of 4 bytes]: the scales, of the activations' type, of rows r and r + 8, which a lane of an mma.sync
//          fragment owns; where the weights have zero points entries of 8 bytes, the second word with the two zero points in its
//          halves.  Without zero points the codes are stored plus 8, and 8 is the zero.  A group of more than 128 columns has its
//          entries in each of its blocks.
// Columns beyond K meet zeros of x and hold code 0, rows beyond O too; the steps of groups and rows that do not exist are zero.
#pragma once
#include <cuda.h>

#include "common.cuh"

namespace bs {

constexpr int W4_ROWS = 16, W4_COLS = 128, W4_CODES = W4_ROWS * W4_COLS / 2;     // bytes of a block's codes
constexpr int W4_MAX_DIM = 1 << 20;     // rows, columns and columns of a group

struct W4Layout {
    int O, K, group, zeros;     // zeros: the matrix has zero points
    int rbs, cbs;               // blocks of rows, blocks of columns
    int block;                  // bytes of a block
    __host__ __device__ size_t bytes() const { return static_cast<size_t>(rbs) * cbs * block; }
};

// Groups of 32 or 64 columns, or a multiple of 128: a block of columns then holds 4, 2 or 1 of them (or a part of one).
inline bool w4_group_ok(int group) { return group == 32 || group == 64 || (group > 0 && group <= W4_MAX_DIM && group % 128 == 0); }

inline bool w4_layout(int O, int K, int group, int zeros, W4Layout& l)
{
    if (O <= 0 || K <= 0 || O > W4_MAX_DIM || K > W4_MAX_DIM || !w4_group_ok(group)) return false;
    l.O = O; l.K = K; l.group = group; l.zeros = zeros != 0;
    l.rbs = ceil_div(O, W4_ROWS); l.cbs = ceil_div(K, W4_COLS);
    l.block = W4_CODES + (group < W4_COLS ? W4_COLS / group : 1) * (zeros ? 64 : 32);
    return true;
}

// The arguments of a product, as every kernel of it takes them.
struct W4Gemm {
    const void* x;              // [M] rows of K values, `ldx` apart
    const unsigned char* w;     // prepared matrix
    const void* bias;           // [O] or null
    void* y;                    // [M] rows of O values, `ldy` apart
    long long ldx, ldy;
    int M;
    W4Layout l;
    int* status;                // device status word
};

// csrc/w4_mma.cu: tensor map of `matrices` prepared matrices, fetched in boxes of `wide` neighbouring blocks of `high` rows of blocks: coordinates (0, block,
// row of blocks, matrix), blocks that do not exist are zeros.
bool w4_encode_blocks(CUtensorMap* tm, const void* prepared, const W4Layout& l, int matrices, int wide, int high);
// Warps of a team, which share a reduction of so many blocks: the widest that leaves at most a fifth of its turns empty, or else the one that leaves the
// fewest.  Wide teams read the weights in long pieces: eight teams of one warp, blocks of 1 KB from eight places, take 1.1 to 1.3 times the time.
inline int w4_team_width(int warps, int blocks)
{
    int best = warps;
    double used = 0;
    for (int split = warps; split >= 1 && used < 0.8; split /= 2) {
        const double u = static_cast<double>(blocks) / (ceil_div(blocks, split) * split);
        if (u > used) { best = split; used = u; }
    }
    return best;
}
// csrc/w4_mma.cu: the product on tcgen05 for many rows of x, which start on 16-byte boundaries.  part: w4_mma_workspace bytes.
bool w4_mma_wanted(int M, const W4Layout& l, int sms);
size_t w4_mma_workspace(int M, const W4Layout& l, int sms);
int w4_mma_launch(const W4Gemm& g, bool f16, float* part, int sms, cudaStream_t st);

}  // namespace bs
