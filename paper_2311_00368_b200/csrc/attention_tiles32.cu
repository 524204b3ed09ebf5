// Launches of the tensor-core attention kernels on fp32 operands: planes, shares, tensor maps.
#include "attention_tiles32.cuh"

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>

#include "attention_maps.h"

namespace b2sp {
namespace attn {
namespace {

constexpr int kBlockCost = 1;   // 1501 x 2903, six heads, 12%: 0, 1, 2, 4 give 63.5, 59.0, 62.6, 64.9 us forward and 184, 185, 190, 201 backward

// Where things lie in the workspace from offset `at` on, and how tiles are dealt out: [0] forward and dQ (by rows), [1] dK and dV (by columns).
struct Plan32 {
    long long tiles[2], blocks[2];
    int outers[2], NB[2], share[2], ctas[2], per[2];
    size_t starts[2], first[2], bad[2], part[2], q, k, v, dout, ml, scores[2], bytes;
    int chunks;
};
Plan32 plan32(const Shape &s, long long tiles, size_t at, bool backward)
{
    Plan32 p = {};
    auto take = [&](size_t b) { const size_t a = at; at += up256(b); return a; };
    p.chunks = (s.d + kPlane - 1) / kPlane;
    const size_t row = p.chunks * kPlanes * 2, qs = (size_t)s.batch * s.heads * s.M, ks = (size_t)s.batch * s.kv_heads * s.K;
    p.q = take(qs * row);
    p.k = take(ks * row);
    p.v = take(ks * row);
    p.dout = take(backward ? qs * row : 0);
    for (int k = 0; k < (backward ? 2 : 1); ++k) {
        p.tiles[k] = tiles * ((long long)s.batch * s.heads / s.patterns);
        p.outers[k] = s.batch * (k == 0 ? s.heads : s.kv_heads);
        p.NB[k] = ((k == 0 ? s.M : s.K) + kTile - 1) / kTile;
        p.blocks[k] = (long long)p.outers[k] * p.NB[k];
        // Equal shares for all SMs; where a block's tiles are few that would leave more sums to join (0.7 us each, one after the other) than
        // it saves tiles (4 us each): not below the square root of a sixth of a block's tiles.
        const long long least = (long long)std::sqrt((double)p.tiles[k] / std::max(1ll, p.blocks[k]) / 6);
        const Shares x = deal(p.tiles[k], p.blocks[k], kBlockCost, least);
        p.per[k] = x.per; p.share[k] = x.share; p.ctas[k] = x.ctas;
        p.starts[k] = take((size_t)p.ctas[k] * 16);
        p.first[k] = take((size_t)(p.ctas[k] + 1) * 8);
        p.bad[k] = take(backward ? (size_t)p.blocks[k] * 4 : 0);
        p.part[k] = take(backward ? (size_t)p.ctas[k] * 2 * (k + 1) * kTile * 64 * 4 : 0);
    }
    if (!backward) {
        const size_t parts = (size_t)(p.ctas[0] + p.blocks[0]) * Fwd32::SETS * kTile;
        p.ml = take(parts * 8);
        p.part[0] = take(parts * 64 * 4);
    }
    for (int k = 0; k < 2; ++k) p.scores[k] = take(p.chunks > 1 && (backward || k == 0) ? (size_t)p.tiles[0] * kScores * 4 : 0);
    p.bytes = at;
    return p;
}

Tiles tiles_of(const Call32 &c, const Plan32 &p, int k)
{
    const Shape &s = c.s;
    return Tiles{k == 0 ? c.plan.rb_ptr : c.plan.cb_ptr, p.NB[k], k == 0 ? s.heads : s.kv_heads, k == 0 ? 1 : s.heads / s.kv_heads, s.patterns, s.batch, s.heads, p.outers[k], p.per[k]};
}

Args32 args(const Call32 &c, const Plan32 &p, int k)
{
    char *ws = static_cast<char *>(c.workspace);
    Args32 f = {};
    RowArgs<float> &r = f.g.a.g;
    r.s = c.s;
    r.ptr = c.row_ptr; r.idx = c.col_idx; r.ptr_stride = c.row_ptr_stride; r.idx_stride = c.nnz_stride;
    r.q = c.q; r.k = c.k; r.v = c.v; r.dout = c.dout;
    r.stat = c.stat; r.stat_stride = c.stat_stride;
    r.lse = c.lse; r.lse_head = c.s.M; r.lse_row = 1;
    r.splits = 1;
    r.fours_in = c.wide_in;
    f.g.a.plan = c.plan;
    f.g.a.col_ptr = c.plan.col_ptr; f.g.a.row_idx = c.plan.row_idx;
    f.g.a.status = c.status;
    f.g.w = tiles_of(c, p, k);
    f.g.tile_at = k == 0 ? c.plan.tile_cb : reinterpret_cast<const int *>(c.plan.ctile);
    f.g.share = p.share[k]; f.g.ctas = p.ctas[k];
    f.g.first = reinterpret_cast<long long *>(ws + p.first[k]);
    f.g.starts = reinterpret_cast<int4 *>(ws + p.starts[k]);
    f.g.bad = reinterpret_cast<int *>(ws + p.bad[k]);
    f.g.part = reinterpret_cast<float *>(ws + p.part[k]);
    f.part_ml = reinterpret_cast<float2 *>(ws + p.ml);
    f.wide = c.wide;
    f.rows = tiles_of(c, p, 0);
    for (int i = 0; i < 2; ++i) f.scores[i] = reinterpret_cast<float *>(ws + p.scores[i]);
    f.dc = c.s.d;
    return f;
}

bool planes_map(CUtensorMap *tm, const Call32 &c, const Plan32 &p, size_t at, int heads, int rows, int box)
{
    const long long row = p.chunks * kPlanes;
    const View<const Bf16> x{reinterpret_cast<const Bf16 *>(static_cast<char *>(c.workspace) + at), row, rows * row, heads * rows * row};
    Op op;
    return make_map(tm, x, c.s.batch, heads, rows, (int)row, box, &op);
}

// Planes of the operands, and where the shares begin.
b2sp_status split(const Call32 &c, const Plan32 &p, bool backward, cudaStream_t st, int *launches)
{
    const Shape &s = c.s;
    char *ws = static_cast<char *>(c.workspace);
    SplitArgs a = {};
    a.d = s.d; a.batch = s.batch; a.chunks = p.chunks;
    auto add = [&](const View<const float> &x, size_t at, int heads, int rows) {
        const int t = a.count++;
        a.x[t] = x; a.planes[t] = reinterpret_cast<Bf16 *>(ws + at); a.heads[t] = heads; a.rows[t] = rows;
        a.before[t + 1] = a.before[t] + (long long)s.batch * heads * rows;
    };
    add(c.q, p.q, s.heads, s.M);
    add(c.k, p.k, s.kv_heads, s.K);
    add(c.v, p.v, s.kv_heads, s.K);
    if (backward) add(c.dout, p.dout, s.heads, s.M);
    ShareArgsOf<float> h = {};
    h.kinds = backward ? 2 : 1;
    long long most = 1;
    for (int k = 0; k < h.kinds; ++k) {
        h.w[k] = tiles_of(c, p, k);
        h.share[k] = p.share[k]; h.ctas[k] = p.ctas[k]; h.rows[k] = k == 0 ? s.M : s.K;
        h.starts[k] = reinterpret_cast<int4 *>(ws + p.starts[k]);
        h.first[k] = reinterpret_cast<long long *>(ws + p.first[k]); h.tiles[k] = p.tiles[k];
        h.bad[k] = backward ? reinterpret_cast<int *>(ws + p.bad[k]) : nullptr;
        most = std::max(most, std::max(p.blocks[k], (long long)p.ctas[0] + p.ctas[1] + 2));
    }
    h.out[0] = c.dq; h.out[1] = c.dk; h.out[2] = c.dv;
    const int share_blocks = (int)((most + 255) / 256);
    const int in_cta = 16 / p.chunks;
    const long long blocks = (a.before[a.count] + in_cta - 1) / in_cta + share_blocks;
    if (blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    if (c.wide_in) split_planes_kernel<4><<<(unsigned)blocks, 256, 0, st>>>(a, h, share_blocks, c.status);
    else split_planes_kernel<1><<<(unsigned)blocks, 256, 0, st>>>(a, h, share_blocks, c.status);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}

// S = Q K^T or dP = dO V^T of all tiles.
b2sp_status product(const Call32 &c, const Plan32 &p, int which, cudaStream_t st, int *launches)
{
    static std::atomic<unsigned long long> done{0};
    const Shape &s = c.s;
    if (p.ctas[0] == 0) return B2SP_OK;
    const Args32 f = args(c, p, 0);
    CUtensorMap x, y;
    if (!planes_map(&x, c, p, which ? p.dout : p.q, s.heads, s.M, 128) || !planes_map(&y, c, p, which ? p.v : p.k, s.kv_heads, s.K, 64) ||
        !allow_smem(tile_product32_kernel, Prod32::BYTES, done))
        return B2SP_ERR_CUDA;
    launch_behind_smem(tile_product32_kernel, (unsigned)p.ctas[0], Prod32::THREADS, Prod32::BYTES, st, x, y, f, f.scores[which]);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}

template <int MODE, bool READ> b2sp_status grad(const Call32 &c, const Plan32 &p, const Args32 &f, cudaStream_t st, int *launches)
{
    static std::atomic<unsigned long long> done{0};
    using C = Grad32<MODE, READ>;
    const Shape &s = c.s;
    CUtensorMap x1, x2, y1, y2;
    const bool q = MODE == kDq;
    const int bq = q ? 128 : 64, bk = q ? 64 : 128;
    if (!planes_map(q ? &x1 : &y1, c, p, p.q, s.heads, s.M, bq) || !planes_map(q ? &x2 : &y2, c, p, p.dout, s.heads, s.M, bq) ||
        !planes_map(q ? &y1 : &x1, c, p, p.k, s.kv_heads, s.K, bk) || !planes_map(q ? &y2 : &x2, c, p, p.v, s.kv_heads, s.K, bk) ||
        !allow_smem(tile_grad32_kernel<MODE, READ>, C::BYTES, done))
        return B2SP_ERR_CUDA;
    launch_behind_smem(tile_grad32_kernel<MODE, READ>, (unsigned)p.ctas[MODE], C::THREADS, C::BYTES, st, x1, x2, y1, y2, f);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}
template <bool READ> b2sp_status backward(const Call32 &c, const Plan32 &p, int col0, cudaStream_t st, int *launches)
{
    constexpr int DW = READ ? 128 : 64;
    const Shape &s = c.s;
    if (p.ctas[0] == 0) return B2SP_OK;   // (both have CTAs, or neither)
    Args32 f[2] = {args(c, p, 0), args(c, p, 1)};
    for (Args32 &x : f) {
        x.col0 = col0;
        x.dc = std::min(kPlane, s.d - col0);
    }
    f[0].g.a.g.out1 = c.dq; f[0].g.a.g.rows = s.M;
    f[1].g.a.g.out1 = c.dk; f[1].g.a.g.out2 = c.dv; f[1].g.a.g.rows = s.K;
    b2sp_status rc = grad<kDq, READ>(c, p, f[0], st, launches);
    if (rc == B2SP_OK) rc = grad<kDkv, READ>(c, p, f[1], st, launches);
    if (rc != B2SP_OK) return rc;
    const unsigned joins = (unsigned)((p.ctas[0] + p.ctas[1]) * kJoinParts);
    if (c.wide) launch_behind(tile_grad_join_kernel<64, float, 4, DW>, joins, 256, st, f[0].g, f[1].g, col0, f[0].dc);
    else launch_behind(tile_grad_join_kernel<64, float, 1, DW>, joins, 256, st, f[0].g, f[1].g, col0, f[0].dc);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}
template <bool READ> b2sp_status forward(const Call32 &c, const Plan32 &p, int col0, cudaStream_t st, int *launches)
{
    static std::atomic<unsigned long long> done{0};
    constexpr int DW = READ ? 128 : 64;
    const Shape &s = c.s;
    Args32 f = args(c, p, 0);
    f.g.a.g.out1 = c.out; f.g.a.g.rows = s.M;
    f.col0 = col0;
    f.dc = std::min(kPlane, s.d - col0);
    CUtensorMap q, k, v;
    if (!planes_map(&q, c, p, p.q, s.heads, s.M, 128) || !planes_map(&k, c, p, p.k, s.kv_heads, s.K, 64) || !planes_map(&v, c, p, p.v, s.kv_heads, s.K, 64) ||
        !allow_smem(tile_forward32_kernel<READ>, Fwd32::BYTES, done))
        return B2SP_ERR_CUDA;
    if (p.ctas[0]) {
        launch_behind_smem(tile_forward32_kernel<READ>, (unsigned)p.ctas[0], Fwd32::THREADS, Fwd32::BYTES, st, q, k, v, f);
        ++*launches;
    }
    const unsigned joins = (unsigned)(p.blocks[0] * kJoinParts32);
    if (c.wide) launch_behind(tile_forward32_join_kernel<4, DW>, joins, 256, st, f);
    else launch_behind(tile_forward32_join_kernel<1, DW>, joins, 256, st, f);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}

}  // namespace

// Widths above 64 keep S (and dP) of all tiles in the workspace: up to 2 GB of them.
bool tiles32_possible(const Shape &s, long long tiles, bool backward)
{
    if (s.d > kMaxTileHeadDim || !(s.scale > 0.f) || !(s.scale <= 3.4e38f) || s.M <= 0 || s.K <= 0) return false;
    return s.d <= kPlane || tiles * ((long long)s.batch * s.heads / s.patterns) * kScores * (backward ? 8 : 4) <= 1ll << 31;
}
size_t tiles32_bytes(const Shape &s, long long tiles, size_t at, bool backward)
{
    return tiles32_possible(s, tiles, backward) ? plan32(s, tiles, at, backward).bytes : at;
}

b2sp_status tiles32_forward(const Call32 &c, cudaStream_t st, int *launches)
{
    const Plan32 p = plan32(c.s, c.tiles, c.scratch_at, false);
    if (p.blocks[0] > INT_MAX / kJoinParts32) return B2SP_ERR_UNSUPPORTED;
    b2sp_status rc = split(c, p, false, st, launches);
    if (p.chunks == 1) return rc == B2SP_OK ? forward<false>(c, p, 0, st, launches) : rc;
    if (rc == B2SP_OK) rc = product(c, p, 0, st, launches);
    for (int k = 0; k < p.chunks && rc == B2SP_OK; ++k) rc = forward<true>(c, p, k * kPlane, st, launches);
    return rc;
}

b2sp_status tiles32_backward(const Call32 &c, cudaStream_t st, int *launches)
{
    const Plan32 p = plan32(c.s, c.tiles, c.scratch_at, true);
    if (p.blocks[0] > INT_MAX / 4 || p.blocks[1] > INT_MAX / 4) return B2SP_ERR_UNSUPPORTED;
    b2sp_status rc = split(c, p, true, st, launches);
    if (p.chunks == 1) return rc == B2SP_OK ? backward<false>(c, p, 0, st, launches) : rc;
    for (int k = 0; k < 2 && rc == B2SP_OK; ++k) rc = product(c, p, k, st, launches);
    for (int k = 0; k < p.chunks && rc == B2SP_OK; ++k) rc = backward<true>(c, p, k * kPlane, st, launches);
    return rc;
}

}  // namespace attn
}  // namespace b2sp
