// Attention over a CSR pattern: what its kernels, its dispatch and its entry points share.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/b2sp.h"

namespace b2sp {
namespace attn {

constexpr int kTile = 128;            // rows and columns of a tile of the pattern
constexpr int kMaxHeadDim = 256;      // row kernels
constexpr int kMaxTileHeadDim = 128;  // tensor-core kernels
constexpr int kMaxColBlocks = 32768;  // 128-column blocks a plan handles (4.2 million columns)
constexpr int kMostPlanRows = 0x7fffffff - (kTile - 1);   // rows a plan handles: the end of the last row block is an int
constexpr int kWarps = 4;             // warps per CTA of the row kernels

// An operand seen as [batch][heads][rows][d].
template <typename T> struct View {
    T *p;
    long long ld, sh, sb;
    __host__ __device__ T *at(int b, int h, long long row) const { return p + b * sb + h * sh + row * ld; }
};

struct Shape {
    int batch, heads, kv_heads, M, K, d, patterns;
    float scale;
};

// Which pattern problem (b, h) has: one for all, one per sequence or one per problem.
__host__ __device__ inline int pattern_of(int patterns, int batch, int heads, int b, int h)
{
    return patterns == 1 ? 0 : patterns == batch ? b : b * heads + h;
}

// Device addresses of a plan's parts (byte offsets from its start; every part begins on 256 bytes).
struct PlanLayout {
    int patterns, M, K, RB, CB, words;   // words: 32-bit words of a row block's bitmap of column blocks
    long long tiles, nnz_stride;
    size_t bitmap, rank, rb_ptr, cb_ptr, tile_cb, ctile, masks, tmasks, col_ptr, row_idx, bytes;
};
inline size_t up256(size_t x) { return (x + 255) & ~size_t(255); }
inline PlanLayout plan_layout(int patterns, int M, int K, long long nnz_stride, long long tiles)
{
    PlanLayout l;
    l.patterns = patterns; l.M = M; l.K = K; l.tiles = tiles; l.nnz_stride = nnz_stride;
    l.RB = (int)((M + (kTile - 1ll)) / kTile);
    l.CB = (int)((K + (kTile - 1ll)) / kTile);
    l.words = (l.CB + 31) / 32;
    const size_t P = patterns, rbs = P * l.RB, cbs = P * l.CB, T = tiles;
    size_t at = 256;   // header: word 0 = flags
    auto take = [&](size_t bytes) { const size_t a = at; at += up256(bytes); return a; };
    l.bitmap = take(rbs * l.words * 4);
    l.rank = take(rbs * l.words * 4);
    l.rb_ptr = take((rbs + 1) * 4);
    l.cb_ptr = take((cbs + 1) * 4);
    l.tile_cb = take(T * 4);
    l.ctile = take(T * 8);
    l.masks = take(T * kTile * 16);
    l.tmasks = take(T * kTile * 16);
    l.col_ptr = take(P * ((size_t)K + 1) * 4);
    l.row_idx = take(P * (size_t)nnz_stride * 4);
    l.bytes = at;
    return l;
}

// What the kernels read of a plan.
struct Plan {
    const int *rb_ptr, *cb_ptr, *tile_cb;
    const int2 *ctile;           // (row block, tile) in the order of the column blocks
    const uint4 *masks, *tmasks; // per tile and row (column): 128 bits
    const int *col_ptr, *row_idx;
    int RB, CB;
};
inline Plan plan_view(const void *plan, const PlanLayout &l)
{
    const char *p = static_cast<const char *>(plan);
    Plan v;
    v.rb_ptr = (const int *)(p + l.rb_ptr);
    v.cb_ptr = (const int *)(p + l.cb_ptr);
    v.tile_cb = (const int *)(p + l.tile_cb);
    v.ctile = (const int2 *)(p + l.ctile);
    v.masks = (const uint4 *)(p + l.masks);
    v.tmasks = (const uint4 *)(p + l.tmasks);
    v.col_ptr = (const int *)(p + l.col_ptr);
    v.row_idx = (const int *)(p + l.row_idx);
    v.RB = l.RB;
    v.CB = l.CB;
    return v;
}
constexpr int kPlanBadColumn = 1, kPlanDuplicate = 2;   // bits of a plan's flag word

}  // namespace attn
}  // namespace b2sp
