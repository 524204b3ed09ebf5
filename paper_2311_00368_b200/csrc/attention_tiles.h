// Interface between the attention entry points and the tensor-core kernels.
#pragma once
#include <algorithm>

#include "attention_rows.cuh"

namespace b2sp {
namespace attn {

// How tiles are dealt to CTAs, one per SM: equal shares of what tiles and blocks cost, a block `cost` tiles ahead of its own, but a quarter
// of the average block at most (blocks without tiles cost nothing in truth); `least`: the smallest share.
struct Shares { int per, share, ctas; };
inline Shares deal(long long tiles, long long blocks, int cost, long long least)
{
    constexpr int kSMs = 148;
    Shares x;
    x.per = (int)std::min((long long)cost, tiles / std::max(1ll, 4 * blocks));
    const long long total = tiles ? tiles + x.per * blocks : 0;
    x.share = (int)std::max(std::max(least, 1ll), (total + kSMs - 1) / kSMs);
    x.ctas = (int)((total + x.share - 1) / x.share);
    return x;
}

// The bfloat16 forward pass: parts of a row block's tiles, up to two CTAs per SM and four tiles a part, where the tiles that a CTA is spared (1.3 us
// each) are worth more than writing and joining the parts.  128 blocks of 32 tiles, width 64, in two parts: 48 -> 36 us; of 16 tiles 27 -> 28, at
// width 128 28 -> 38 us.
struct FwdSplit { int splits; double cost; };   // us
inline FwdSplit tile_splits(const Shape &s, long long tiles)
{
    const long long blocks = std::max(1ll, (long long)s.batch * s.heads * ((s.M + kTile - 1) / kTile));
    const long long in_block = tiles * ((long long)s.batch * s.heads / s.patterns) / blocks;
    const long long splits = std::min(2 * 148 / blocks, in_block / 4);
    if (splits < 2) return {1, 0};
    const double cost = 6 + blocks * splits / 256.0 * (s.d <= 64 ? 5 : 14);
    if (1.3 * (in_block - in_block / splits) < cost) return {1, 0};
    return {(int)splits, cost};
}

struct TileCall {
    Shape s;
    Plan plan;
    long long tiles;                     // of all patterns
    const int *row_ptr, *col_idx;        // for rows that have to be taken one by one (see attention_tiles.cuh)
    long long row_ptr_stride, nnz_stride;
    View<const Bf16> q, k, v, dout, o;   // o: the forward pass's result, in the backward pass
    View<Bf16> out, dq, dk, dv;
    float *lse;                          // backward: read
    const float2 *stat;
    long long stat_stride;
    int *status;
    void *workspace;
    size_t scratch_at;                   // where the workspace is free
};

bool tiles_possible(const Shape &s, const View<const Bf16> *views, int n);
// The end of what a pass needs of the workspace, from offset `at` on.
size_t tiles_bytes(const Shape &s, long long tiles, size_t at, bool backward);
b2sp_status tiles_forward(const TileCall &c, cudaStream_t st, int *launches);
b2sp_status tiles_backward(const TileCall &c, cudaStream_t st, int *launches);

// The same on fp32 operands, of any alignment.
struct Call32 {
    Shape s;
    Plan plan;
    long long tiles;
    const int *row_ptr, *col_idx;
    long long row_ptr_stride, nnz_stride;
    View<const float> q, k, v, dout;
    View<float> out, dq, dk, dv;
    int wide_in, wide;                   // all inputs (outputs) have rows that are aligned groups of four elements
    float *lse;
    const float2 *stat;
    long long stat_stride;
    int *status;
    void *workspace;
    size_t scratch_at;
};
bool tiles32_possible(const Shape &s, long long tiles, bool backward);
size_t tiles32_bytes(const Shape &s, long long tiles, size_t at, bool backward);
b2sp_status tiles32_forward(const Call32 &c, cudaStream_t st, int *launches);
b2sp_status tiles32_backward(const Call32 &c, cudaStream_t st, int *launches);

}  // namespace attn
}  // namespace b2sp
