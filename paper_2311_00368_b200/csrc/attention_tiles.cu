// Launches of the tensor-core attention kernels: tensor maps, grids.
#include "attention_tiles.cuh"

#include "attention_maps.h"

#include <algorithm>
#include <atomic>
#include <climits>
#include <mutex>

namespace b2sp {
namespace attn {
namespace {

constexpr int kBlockCost = 2;   // tiles that a block's start and end take: under a window 0, 2, 4 give 339, 322, 322 us; with blocks of equal length no difference

TileArgs args(const TileCall &c)
{
    TileArgs a = {};
    a.g.s = c.s;
    a.g.ptr = c.row_ptr; a.g.idx = c.col_idx; a.g.ptr_stride = c.row_ptr_stride; a.g.idx_stride = c.nnz_stride;
    a.g.q = c.q; a.g.k = c.k; a.g.v = c.v; a.g.dout = c.dout;
    a.g.stat = c.stat; a.g.stat_stride = c.stat_stride;
    a.g.lse = c.lse; a.g.lse_head = c.s.M; a.g.lse_row = 1;
    a.g.splits = 1;
    a.plan = c.plan;
    a.col_ptr = c.plan.col_ptr; a.row_idx = c.plan.row_idx;
    a.status = c.status;
    return a;
}

struct FwdPlan { int splits; size_t part, ml, bytes; };   // offsets
FwdPlan forward_plan(const Shape &s, long long tiles, size_t at)
{
    FwdPlan p;
    const long long blocks = (long long)s.batch * s.heads * ((s.M + kTile - 1) / kTile);
    p.splits = tile_splits(s, tiles).splits;
    p.part = at;
    p.ml = at + (p.splits > 1 ? (size_t)blocks * p.splits * kTile * (s.d <= 64 ? 64 : 128) * 4 : 0);
    p.bytes = p.ml + up256(p.splits > 1 ? (size_t)blocks * p.splits * kTile * 8 : 0);
    return p;
}
template <int DP, bool SPLIT> b2sp_status launch_forward(const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, const TileArgs &a, const FwdParts &f, unsigned ctas, cudaStream_t st)
{
    static std::atomic<unsigned long long> done{0};
    if (!allow_smem(tile_forward_kernel<DP, SPLIT>, FwdCfg<DP>::BYTES, done)) return B2SP_ERR_CUDA;
    tile_forward_kernel<DP, SPLIT><<<ctas, kTileThreads, FwdCfg<DP>::BYTES, st>>>(q, k, v, a, f);
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}
template <int DP> b2sp_status forward(const TileCall &c, cudaStream_t st, int *launches)
{
    TileArgs a = args(c);
    a.g.out1 = c.out; a.g.rows = c.s.M;
    CUtensorMap q, k, v;
    if (!make_map(&q, c.q, c.s.batch, c.s.heads, c.s.M, c.s.d, 128, &a.q) || !make_map(&k, c.k, c.s.batch, c.s.kv_heads, c.s.K, c.s.d, 64, &a.k) ||
        !make_map(&v, c.v, c.s.batch, c.s.kv_heads, c.s.K, c.s.d, 64, &a.v))
        return B2SP_ERR_CUDA;
    const FwdPlan p = forward_plan(c.s, c.tiles, c.scratch_at);
    const long long blocks = (long long)c.s.batch * c.s.heads * c.plan.RB;
    if (blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    char *ws = static_cast<char *>(c.workspace);
    const FwdParts f{p.splits, reinterpret_cast<float *>(ws + p.part), reinterpret_cast<float2 *>(ws + p.ml)};
    ++*launches;
    if (p.splits == 1) return launch_forward<DP, false>(q, k, v, a, f, (unsigned)blocks, st);
    const b2sp_status rc = launch_forward<DP, true>(q, k, v, a, f, (unsigned)(blocks * p.splits), st);
    if (rc != B2SP_OK) return rc;
    launch_behind(tile_forward_join_kernel<DP>, (unsigned)(blocks * (kTile * DP / 4 / 256)), 256, st, a, f);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}

// How the backward pass is dealt out: shares of tiles for dQ (0) and for dK and dV (1), and where things lie in the workspace.
struct GradPlan {
    long long tiles[2];
    int outers[2], NB[2], share[2], ctas[2];
    int per[2];
    size_t starts[2], first[2], bad[2], part[2], bytes;
};
GradPlan grad_plan(const Shape &s, long long tiles, size_t at)
{
    GradPlan p;
    const int DP = s.d <= 64 ? 64 : 128;
    for (int k = 0; k < 2; ++k) {
        p.tiles[k] = tiles * ((long long)s.batch * s.heads / s.patterns);
        p.outers[k] = s.batch * (k == 0 ? s.heads : s.kv_heads);
        p.NB[k] = ((k == 0 ? s.M : s.K) + kTile - 1) / kTile;
        const Shares x = deal(p.tiles[k], (long long)p.outers[k] * p.NB[k], kBlockCost, 1);
        p.per[k] = x.per; p.share[k] = x.share; p.ctas[k] = x.ctas;
        p.starts[k] = at;
        at += up256((size_t)p.ctas[k] * 16);
        p.first[k] = at;
        at += up256((size_t)(p.ctas[k] + 1) * 8);
        p.bad[k] = at;
        at += up256((size_t)p.outers[k] * p.NB[k] * 4);
        p.part[k] = at;
        at += (size_t)p.ctas[k] * 2 * (k + 1) * kTile * DP * 4;
    }
    p.bytes = at;
    return p;
}

template <int MODE, int DP> b2sp_status grad(const TileCall &c, const GradPlan &p, GradArgs &g, cudaStream_t st, int *launches)
{
    static std::atomic<unsigned long long> done{0};
    using C = GradCfg<MODE, DP>;
    const Shape &s = c.s;
    CUtensorMap x1, x2, y1, y2;
    const bool q = MODE == kDq;
    const int box_q = q ? 128 : 64, box_k = q ? 64 : 128;
    if (!make_map(q ? &x1 : &y1, c.q, s.batch, s.heads, s.M, s.d, box_q, &g.a.q) || !make_map(q ? &x2 : &y2, c.dout, s.batch, s.heads, s.M, s.d, box_q, &g.a.dout) ||
        !make_map(q ? &y1 : &x1, c.k, s.batch, s.kv_heads, s.K, s.d, box_k, &g.a.k) || !make_map(q ? &y2 : &x2, c.v, s.batch, s.kv_heads, s.K, s.d, box_k, &g.a.v) ||
        !allow_smem(tile_grad_kernel<MODE, DP>, C::BYTES, done))
        return B2SP_ERR_CUDA;
    if (g.ctas) {
        launch_behind_smem(tile_grad_kernel<MODE, DP>, (unsigned)g.ctas, C::THREADS, C::BYTES, st, x1, x2, y1, y2, g);
        ++*launches;
    }
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}

template <int DP> b2sp_status backward(const TileCall &c, cudaStream_t st, int *launches)
{
    const Shape &s = c.s;
    const GradPlan p = grad_plan(s, c.tiles, c.scratch_at);
    char *ws = static_cast<char *>(c.workspace);
    if ((long long)p.outers[0] * p.NB[0] > INT_MAX / 4 || (long long)p.outers[1] * p.NB[1] > INT_MAX / 4) return B2SP_ERR_UNSUPPORTED;
    GradArgs g[2] = {};
    ShareArgs h = {};
    h.kinds = 2;
    for (int k = 0; k < 2; ++k) {
        g[k].a = args(c);
        g[k].w = Tiles{k == 0 ? c.plan.rb_ptr : c.plan.cb_ptr, p.NB[k], k == 0 ? s.heads : s.kv_heads, k == 0 ? 1 : s.heads / s.kv_heads, s.patterns, s.batch, s.heads, p.outers[k], p.per[k]};
        g[k].tile_at = k == 0 ? c.plan.tile_cb : reinterpret_cast<const int *>(c.plan.ctile);
        g[k].share = p.share[k]; g[k].ctas = p.ctas[k];
        g[k].first = reinterpret_cast<long long *>(ws + p.first[k]);
        g[k].starts = reinterpret_cast<int4 *>(ws + p.starts[k]);
        g[k].bad = reinterpret_cast<int *>(ws + p.bad[k]);
        g[k].part = reinterpret_cast<float *>(ws + p.part[k]);
        h.w[k] = g[k].w; h.share[k] = p.share[k]; h.ctas[k] = p.ctas[k]; h.rows[k] = k == 0 ? s.M : s.K;
        h.starts[k] = reinterpret_cast<int4 *>(ws + p.starts[k]); h.bad[k] = g[k].bad;
        h.first[k] = reinterpret_cast<long long *>(ws + p.first[k]); h.tiles[k] = p.tiles[k];
    }
    g[0].a.g.out1 = c.dq; g[0].a.g.rows = s.M;
    g[1].a.g.out1 = c.dk; g[1].a.g.out2 = c.dv; g[1].a.g.rows = s.K;
    h.out[0] = c.dq; h.out[1] = c.dk; h.out[2] = c.dv;
    const long long rows = (long long)s.batch * s.heads * c.stat_stride, blocks = (rows + 16 * kStatRows - 1) / (16 * kStatRows);
    const int share_blocks = (std::max(p.ctas[0] + p.ctas[1] + 2, std::max(p.outers[0] * p.NB[0], p.outers[1] * p.NB[1])) + 255) / 256;
    if (blocks + share_blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    tile_grad_stat_kernel<><<<(unsigned)(blocks + share_blocks), 256, 0, st>>>(s, c.o, c.dout, c.lse, (int)c.stat_stride, const_cast<float2 *>(c.stat), h, share_blocks, c.status);
    ++*launches;
    b2sp_status rc = grad<kDq, DP>(c, p, g[0], st, launches);
    if (rc == B2SP_OK) rc = grad<kDkv, DP>(c, p, g[1], st, launches);
    if (rc != B2SP_OK || p.ctas[0] == 0) return rc;   // (both have CTAs, or neither)
    launch_behind(tile_grad_join_kernel<DP>, (unsigned)((g[0].ctas + g[1].ctas) * kJoinParts), 256, st, g[0], g[1], 0, s.d);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}

// ---- widths that are no multiple of eight --------------------------------------------------------------------------------------------
// Tensor maps want rows of whole 16-byte pieces.  Other widths are copied into the workspace with zeros behind them, which add nothing to a
// product, and results are copied out.  Eight elements a thread, aligned on the wide side, one by one on the other.  At 8 heads of 4096 and
// width 83, 16.5%, forward and backward: 105 and 303 us; the row kernels take 1983 and 6850, width 88 where it lies 91 and 262.
struct CopyArgs {
    View<Bf16> narrow[5], wide[5];
    int heads[5], rows[5], count, d, groups;   // groups of eight in a wide row
    long long before[6];                       // groups of the tensors ahead
};
template <bool IN> __global__ void __launch_bounds__(256) copy_rows_kernel(const __grid_constant__ CopyArgs a)
{
    long long at = blockIdx.x * 256ll + threadIdx.x;
    if (at >= a.before[a.count]) return;
    int t = 0;
    while (t + 1 < a.count && at >= a.before[t + 1]) ++t;
    at -= a.before[t];
    const long long row = at / a.groups;
    const int c = (int)(at % a.groups) * 8, prob = (int)(row / a.rows[t]), b = prob / a.heads[t], h = prob % a.heads[t];
    unsigned short *x = reinterpret_cast<unsigned short *>(a.narrow[t].at(b, h, row % a.rows[t])) + c;
    uint4 *y = reinterpret_cast<uint4 *>(a.wide[t].at(b, h, row % a.rows[t]) + c);
    union { uint4 v; unsigned short e[8]; } u;
    if (!IN) u.v = *y;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (IN) u.e[k] = c + k < a.d ? x[k] : (unsigned short)0;
        else if (c + k < a.d) x[k] = u.e[k];
    }
    if (IN) *y = u.v;
}

struct Staging {
    CopyArgs in = {}, out = {};
    char *ws;
    const Shape &s;
    size_t at;
    Staging(const Shape &s_, char *ws_, size_t at_) : ws(ws_), s(s_), at(at_) {}
    // a place for a tensor of this many heads and rows
    View<Bf16> add(CopyArgs &a, const View<Bf16> &x, int heads, int rows)
    {
        const int D = (s.d + 7) / 8 * 8, t = a.count++;
        const View<Bf16> y{reinterpret_cast<Bf16 *>(ws + at), D, (long long)rows * D, (long long)heads * rows * D};
        at += up256((size_t)s.batch * heads * rows * D * 2);
        a.narrow[t] = x; a.wide[t] = y; a.heads[t] = heads; a.rows[t] = rows;
        a.d = s.d; a.groups = D / 8;
        a.before[t + 1] = a.before[t] + (long long)s.batch * heads * rows * (D / 8);
        return y;
    }
    View<const Bf16> read(const View<const Bf16> &x, int heads, int rows)
    {
        const View<Bf16> y = add(in, View<Bf16>{const_cast<Bf16 *>(x.p), x.ld, x.sh, x.sb}, heads, rows);
        return View<const Bf16>{y.p, y.ld, y.sh, y.sb};
    }
};
// What is staged, from offset c.scratch_at on, which moves behind it; called without a workspace for the size alone.
Staging stage(TileCall &c, bool backward)
{
    const Shape &s = c.s;
    Staging g(s, static_cast<char *>(c.workspace), c.scratch_at);
    c.q = g.read(c.q, s.heads, s.M);
    c.k = g.read(c.k, s.kv_heads, s.K);
    c.v = g.read(c.v, s.kv_heads, s.K);
    if (backward) {
        c.o = g.read(c.o, s.heads, s.M);
        c.dout = g.read(c.dout, s.heads, s.M);
        c.dq = g.add(g.out, c.dq, s.heads, s.M);
        c.dk = g.add(g.out, c.dk, s.kv_heads, s.K);
        c.dv = g.add(g.out, c.dv, s.kv_heads, s.K);
    } else {
        c.out = g.add(g.out, c.out, s.heads, s.M);
    }
    c.scratch_at = g.at;
    return g;
}
template <bool IN> b2sp_status copy(const CopyArgs &a, cudaStream_t st, int *launches)
{
    const long long blocks = (a.before[a.count] + 255) / 256;
    if (blocks == 0) return B2SP_OK;
    if (blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    copy_rows_kernel<IN><<<(unsigned)blocks, 256, 0, st>>>(a);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}
template <class F> b2sp_status staged(TileCall c, bool backward, cudaStream_t st, int *launches, F run)
{
    if (!(c.s.d & 7)) return run(c);
    const Shape s = c.s;
    Staging g = stage(c, backward);
    c.s.d = (s.d + 7) / 8 * 8;
    b2sp_status rc = copy<true>(g.in, st, launches);
    if (rc == B2SP_OK) rc = run(c);
    return rc == B2SP_OK ? copy<false>(g.out, st, launches) : rc;
}

}  // namespace

// Widths up to 128, and a factor that keeps the order of the products (the reference of the exponentials is the largest of them).  Widths in
// whole 16-byte pieces are read where they lie: every address and stride a multiple of 16 bytes.
bool tiles_possible(const Shape &s, const View<const Bf16> *views, int n)
{
    if (s.d > kMaxTileHeadDim || !(s.scale > 0.f) || !(s.scale <= 3.4e38f)) return false;
    if (s.d & 7) return true;
    for (int i = 0; i < n; ++i) {
        const View<const Bf16> &v = views[i];
        if ((reinterpret_cast<uintptr_t>(v.p) & 15) || ((v.ld | v.sh | v.sb) & 7) || v.ld < s.d) return false;
        if (v.ld >= (1ll << 38) || v.sh >= (1ll << 38) || v.sb >= (1ll << 38)) return false;
    }
    return true;
}

size_t tiles_bytes(const Shape &s, long long tiles, size_t at, bool backward)
{
    if (s.d > kMaxTileHeadDim) return at;
    if (s.d & 7) {
        TileCall c = {};
        c.s = s; c.scratch_at = at;
        stage(c, backward);
        at = c.scratch_at;
    }
    return backward ? grad_plan(s, tiles, at).bytes : forward_plan(s, tiles, at).bytes;
}
b2sp_status tiles_forward(const TileCall &c, cudaStream_t st, int *launches)
{
    return staged(c, false, st, launches, [&](const TileCall &x) { return x.s.d <= 64 ? forward<64>(x, st, launches) : forward<128>(x, st, launches); });
}
b2sp_status tiles_backward(const TileCall &c, cudaStream_t st, int *launches)
{
    return staged(c, true, st, launches, [&](const TileCall &x) { return x.s.d <= 64 ? backward<64>(x, st, launches) : backward<128>(x, st, launches); });
}

}  // namespace attn
}  // namespace b2sp
