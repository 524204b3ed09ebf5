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

constexpr int kSMs = 148;

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

template <int DP> b2sp_status forward(const TileCall &c, cudaStream_t st, int *launches)
{
    static std::atomic<unsigned long long> done{0};
    TileArgs a = args(c);
    a.g.out1 = c.out; a.g.rows = c.s.M;
    CUtensorMap q, k, v;
    if (!make_map(&q, c.q, c.s.batch, c.s.heads, c.s.M, c.s.d, 128, &a.q) || !make_map(&k, c.k, c.s.batch, c.s.kv_heads, c.s.K, c.s.d, 64, &a.k) ||
        !make_map(&v, c.v, c.s.batch, c.s.kv_heads, c.s.K, c.s.d, 64, &a.v) || !allow_smem(tile_forward_kernel<DP>, FwdCfg<DP>::BYTES, done))
        return B2SP_ERR_CUDA;
    const long long blocks = (long long)c.s.batch * c.s.heads * c.plan.RB;
    if (blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    tile_forward_kernel<DP><<<(unsigned)blocks, kTileThreads, FwdCfg<DP>::BYTES, st>>>(q, k, v, a);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}

// How the backward pass is dealt out: shares of tiles for dQ (0) and for dK and dV (1), and where things lie in the workspace.
struct GradPlan {
    long long tiles[2];
    int outers[2], NB[2], share[2], ctas[2];
    size_t starts[2], bad[2], part, bytes;   // offsets from `at`
};
GradPlan grad_plan(const Shape &s, long long tiles, size_t at)
{
    GradPlan p;
    const int DP = s.d <= 64 ? 64 : 128;
    size_t part = 0;
    for (int k = 0; k < 2; ++k) {
        p.tiles[k] = tiles * ((long long)s.batch * s.heads / s.patterns);
        p.outers[k] = s.batch * (k == 0 ? s.heads : s.kv_heads);
        p.NB[k] = ((k == 0 ? s.M : s.K) + kTile - 1) / kTile;
        p.share[k] = (int)std::max(1ll, (p.tiles[k] + kSMs - 1) / kSMs);
        p.ctas[k] = (int)((p.tiles[k] + p.share[k] - 1) / p.share[k]);
        p.starts[k] = at;
        at += up256((size_t)p.ctas[k] * 16);
        p.bad[k] = at;
        at += up256((size_t)p.outers[k] * p.NB[k] * 4);
        part = std::max(part, (size_t)p.ctas[k] * 2 * (k + 1) * kTile * DP * 4);
    }
    p.part = at;
    p.bytes = at + up256(part);
    return p;
}

template <int MODE, int DP> b2sp_status grad(const TileCall &c, const GradPlan &p, GradArgs g, cudaStream_t st, int *launches)
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
        launch_behind(tile_grad_join_kernel<MODE, DP>, (unsigned)(g.ctas * kJoinParts), 256, st, g);
        *launches += 2;
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
        g[k].w = Tiles{k == 0 ? c.plan.rb_ptr : c.plan.cb_ptr, p.NB[k], k == 0 ? s.heads : s.kv_heads, k == 0 ? 1 : s.heads / s.kv_heads, s.patterns, s.batch, s.heads, p.outers[k]};
        g[k].tile_at = k == 0 ? c.plan.tile_cb : reinterpret_cast<const int *>(c.plan.ctile);
        g[k].share = p.share[k]; g[k].ctas = p.ctas[k]; g[k].tiles = p.tiles[k];
        g[k].starts = reinterpret_cast<int4 *>(ws + p.starts[k]);
        g[k].bad = reinterpret_cast<int *>(ws + p.bad[k]);
        g[k].part = reinterpret_cast<float *>(ws + p.part);
        h.w[k] = g[k].w; h.share[k] = p.share[k]; h.ctas[k] = p.ctas[k]; h.rows[k] = k == 0 ? s.M : s.K;
        h.starts[k] = reinterpret_cast<int4 *>(ws + p.starts[k]); h.bad[k] = g[k].bad;
    }
    g[0].a.g.out1 = c.dq; g[0].a.g.rows = s.M;
    g[1].a.g.out1 = c.dk; g[1].a.g.out2 = c.dv; g[1].a.g.rows = s.K;
    h.out[0] = c.dq; h.out[1] = c.dk; h.out[2] = c.dv;
    const long long rows = (long long)s.batch * s.heads * c.stat_stride, blocks = (rows + 16 * kStatRows - 1) / (16 * kStatRows);
    const int share_blocks = (std::max(std::max(1, p.ctas[0] + p.ctas[1]), std::max(p.outers[0] * p.NB[0], p.outers[1] * p.NB[1])) + 255) / 256;
    if (blocks + share_blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    tile_grad_stat_kernel<><<<(unsigned)(blocks + share_blocks), 256, 0, st>>>(s, c.o, c.dout, c.lse, (int)c.stat_stride, const_cast<float2 *>(c.stat), h, share_blocks, c.status);
    ++*launches;
    const b2sp_status rc = grad<kDq, DP>(c, p, g[0], st, launches);
    return rc == B2SP_OK ? grad<kDkv, DP>(c, p, g[1], st, launches) : rc;
}

}  // namespace

// Widths up to 128 in whole 16-byte pieces, every address and stride a multiple of 16 bytes, and a factor that keeps the order of the
// products (the reference of the exponentials is the largest of them).
bool tiles_possible(const Shape &s, const View<const Bf16> *views, int n)
{
    if (s.d > kMaxTileHeadDim || (s.d & 7) || !(s.scale > 0.f) || !(s.scale <= 3.4e38f)) return false;
    for (int i = 0; i < n; ++i) {
        const View<const Bf16> &v = views[i];
        if ((reinterpret_cast<uintptr_t>(v.p) & 15) || ((v.ld | v.sh | v.sb) & 7) || v.ld < s.d) return false;
        if (v.ld >= (1ll << 38) || v.sh >= (1ll << 38) || v.sb >= (1ll << 38)) return false;
    }
    return true;
}

size_t tiles_backward_bytes(const Shape &s, long long tiles, size_t at)
{
    return s.d <= kMaxTileHeadDim ? grad_plan(s, tiles, at).bytes : at;
}
b2sp_status tiles_forward(const TileCall &c, cudaStream_t st, int *launches)
{
    return c.s.d <= 64 ? forward<64>(c, st, launches) : forward<128>(c, st, launches);
}
b2sp_status tiles_backward(const TileCall &c, cudaStream_t st, int *launches)
{
    return c.s.d <= 64 ? backward<64>(c, st, launches) : backward<128>(c, st, launches);
}

}  // namespace attn
}  // namespace b2sp
