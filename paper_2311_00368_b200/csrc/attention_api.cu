// Entry points of attention over a CSR pattern: argument checks, plans, choice of the kernel family, launches.  See include/b2sp.h.
#include <algorithm>
#include <climits>

#include "../../include/b2sp_debug.h"
#include "attention_plan.cuh"
#include "attention_rows.cuh"
#include "attention_tiles.h"

namespace b2sp {
namespace attn {

constexpr size_t kHeader = 512;   // of a workspace: int 64 is the status word that b2sp_device_status reads

thread_local int g_algo[2] = {-1, -1}, g_launches[2] = {0, 0};

inline b2sp_status launched() { return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA; }

b2sp_status check_pattern(int patterns, int M, int K, long long nnz_stride, const int *row_ptr, long long row_ptr_stride, const int *col_idx)
{
    if (patterns < 1 || M < 0 || K < 0 || nnz_stride < 0 || nnz_stride > INT_MAX) return B2SP_ERR_INVALID_ARG;
    if ((!row_ptr && M) || (nnz_stride && !col_idx)) return B2SP_ERR_INVALID_ARG;
    if (patterns > 1 && row_ptr_stride < M + 1ll) return B2SP_ERR_INVALID_ARG;
    return B2SP_OK;
}

b2sp_status check_problem(const b2sp_attention_problem *p)
{
    if (!p || p->batch < 1 || p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads || p->d < 1) return B2SP_ERR_INVALID_ARG;
    if ((long long)p->batch * p->heads > INT_MAX) return B2SP_ERR_INVALID_ARG;
    if (p->patterns != 1 && p->patterns != p->batch && p->patterns != p->batch * p->heads) return B2SP_ERR_INVALID_ARG;
    if (!(p->scale == p->scale)) return B2SP_ERR_INVALID_ARG;
    if (p->plan && (p->plan_tiles < 0 || (reinterpret_cast<uintptr_t>(p->plan) & 255))) return B2SP_ERR_INVALID_ARG;
    const b2sp_status rc = check_pattern(p->patterns, p->M, p->K, p->nnz_stride, p->row_ptr, p->row_ptr_stride, p->col_idx);
    if (rc != B2SP_OK) return rc;
    if (p->plan && (p->M > kMostPlanRows || p->K > kMaxColBlocks * kTile)) return B2SP_ERR_UNSUPPORTED;   // (no plan has these sizes)
    return p->d > kMaxHeadDim ? B2SP_ERR_UNSUPPORTED : B2SP_OK;
}

b2sp_status check_operand(const b2sp_heads *x, int rows, int d)
{
    if (!x) return B2SP_ERR_INVALID_ARG;
    if (rows && !x->data) return B2SP_ERR_INVALID_ARG;
    if (rows > 1 && x->ld < 0) return B2SP_ERR_INVALID_ARG;
    if (x->stride_head < 0 || x->stride_batch < 0) return B2SP_ERR_INVALID_ARG;
    return B2SP_OK;
}
// An output: rows do not overlap, and neither do heads and sequences (whichever is the inner one).
b2sp_status check_output(const b2sp_heads *x, int batch, int heads, int rows, int d)
{
    const b2sp_status rc = check_operand(x, rows, d);
    if (rc != B2SP_OK || !rows) return rc;
    if (rows > 1 && x->ld < d) return B2SP_ERR_INVALID_ARG;
    // sorted by stride, every dimension must step over the extent of the smaller ones
    long long stride[3] = {x->ld, x->stride_head, x->stride_batch};
    long long count[3] = {rows, heads, batch};
    long long extent = d;
    for (int i = 0; i < 3; ++i) {
        int k = -1;
        for (int j = 0; j < 3; ++j)
            if (count[j] > 1 && (k < 0 || stride[j] < stride[k])) k = j;
        if (k < 0) break;
        if (stride[k] < extent) return B2SP_ERR_INVALID_ARG;
        extent += stride[k] * (count[k] - 1);
        count[k] = 1;
    }
    return B2SP_OK;
}

template <typename T> View<T> view(const b2sp_heads *x) { return View<T>{static_cast<T *>(x->data), x->ld, x->stride_head, x->stride_batch}; }
Shape shape(const b2sp_attention_problem *p) { return Shape{p->batch, p->heads, p->kv_heads, p->M, p->K, p->d, p->patterns, p->scale}; }

// Whether rows of a view are aligned groups of four elements.
template <typename T> bool fours(const View<T> &v, int d)
{
    return ((reinterpret_cast<uintptr_t>(v.p) / sizeof(T) | (uintptr_t)v.ld | (uintptr_t)v.sh | (uintptr_t)v.sb | (uintptr_t)d) & 3) == 0 &&
           reinterpret_cast<uintptr_t>(v.p) % sizeof(T) == 0;
}

// ---- row kernels: parts of rows and what they leave in the workspace ----------------------------------------------------------------
// Enough warps for every SM to have sixteen, parts of 64 entries at least on average.
int pick_splits(long long rows, long long problems, long long nnz)
{
    const long long units = std::max(1ll, rows * problems), want = 148ll * 16;
    if (units >= want || nnz <= 0) return 1;
    const long long avg = nnz / std::max(1ll, rows);
    return (int)std::max(1ll, std::min((want + units - 1) / units, std::min((long long)4096, avg / 64)));
}
struct RowPlan {
    int splits_m, splits_k;               // of rows and (dK, dV) of columns
    bool parts_kv;
    size_t stat, ml, part, bytes;         // offsets
    int stat_rows;
};
RowPlan row_plan(const Shape &s, long long nnz, bool backward, long long tiles, bool planned, bool fp32)
{
    RowPlan r;
    const long long problems = (long long)s.batch * s.heads;
    r.splits_m = pick_splits(s.M, problems, nnz);
    r.splits_k = pick_splits(s.K, problems, nnz);
    r.stat_rows = backward ? (s.M + kTile - 1) / kTile * kTile : 0;
    r.parts_kv = r.splits_k > 1 || s.heads != s.kv_heads;
    size_t at = kHeader;
    auto take = [&](size_t b) { const size_t a = at; at += up256(b); return a; };
    const size_t um = problems * s.M * r.splits_m, uk = problems * s.K * r.splits_k;
    r.stat = take(backward ? problems * r.stat_rows * 8 : 0);
    r.ml = take(!backward && r.splits_m > 1 ? um * 8 : 0);
    size_t part = r.splits_m > 1 ? um * part_width(kForward, s.d) * 4 : 0;
    if (backward && r.parts_kv) part = std::max(part, uk * part_width(kGradKV, s.d) * 4);
    r.part = take(part);
    r.bytes = at;   // (the tile kernels use what lies behind the statistics)
    if (planned) r.bytes = std::max(r.bytes, fp32 ? tiles32_bytes(s, tiles, r.ml, backward) : tiles_bytes(s, tiles, r.ml, backward));
    return r;
}

template <int MODE, typename T, int V> b2sp_status launch_rows(const RowArgs<T> &g, cudaStream_t st, int *launches)
{
    const long long units = (long long)g.s.batch * g.s.heads * g.rows * g.splits;
    if (units == 0) return B2SP_OK;
    const long long blocks = (units + kWarps - 1) / kWarps;
    if (blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    if (g.s.d <= 64) attention_row_kernel<MODE, T, V, 64><<<(unsigned)blocks, kWarps * 32, 0, st>>>(g);
    else if (g.s.d <= 128) attention_row_kernel<MODE, T, V, 128><<<(unsigned)blocks, kWarps * 32, 0, st>>>(g);
    else attention_row_kernel<MODE, T, V, 256><<<(unsigned)blocks, kWarps * 32, 0, st>>>(g);
    ++*launches;
    if (g.part) {
        if (!launch_join<MODE, T, V>(g, st)) return B2SP_ERR_UNSUPPORTED;
        ++*launches;
    }
    return launched();
}
template <int MODE, typename T> b2sp_status launch_rows_v(bool wide, const RowArgs<T> &g, cudaStream_t st, int *launches)
{
    return wide ? launch_rows<MODE, T, 4>(g, st, launches) : launch_rows<MODE, T, 1>(g, st, launches);
}

// ---- the choice between the families -------------------------------------------------------------------------------------------------
// Microseconds that each would take.  The row kernels' work is that of the stored entries, but a warp takes a row's (or a part's, about 64 and
// more) one after the other.  The tile kernels' work is that of the tiles, whatever they hold; the forward pass takes a block's (or
// a part's) one after the other.  Measured, rows against tiles, bf16, width 64, forward and backward:
//     one row of 4096 of 8192, one head              26 and  32    14 and  30   (87 before long blocks were cut into parts)
//     512 x 512 at 2%, one head                       7 and  15    10 and  28
//     1024 x 1024 at 0.5%, 8 heads                   11 and  27    16 and  45
//     2048 x 2048 at 1%, 8 heads over 2              33 and  81    27 and  78
//     2048 x 2048 at 4%, 8 heads over 2              85 and 212    27 and  78
//     200 x 8000 at 2%, one head                     30 and  38    16 and  46   (85)
//     128 x 8192 at 50%, 8 heads, width 128         400            17          (86)
//     4 x 5 heads over one, width 32, 700 x 700, 3%  28 and  73    13 and  52
//     256 x 256, 12 heads over 3, width 119, 29%     43 and 141    14 and  47
// fp32:
//     one row of 4096 of 8192, one head              26 and  36    36 and  48
//     64 x 64 at 30%, one head                        7 and  17    14 and  30
//     2048 x 2048 at 2%, 8 heads over 2              52 and 156    66 and 204
//     2048 x 2048 at 4%, 8 heads over 2              88 and 267    66 and 205
//     200 x 8000 at 2%, one head                     31 and  47    38 and  58
// fp32, width 128 (see tile_product32_kernel):
//     64 x 64 at 30%, one head                        9 and  24    38 and  82
//     256 x 256 at 29%, 12 heads over 3              31 and 144    42 and 100   (width 120; 119: 43 and 155, 43 and 103)
//     2048 x 2048 at 2%, 8 heads over 2              74 and 283   228 and 733
//     4096 x 4096 at 30%, 8 heads                  2752           751
//     4096 x 4096, window of 1229, 8 heads over 2         9534            928
double row_time(const Shape &s, double entries, double in_row, bool backward, bool fp32)
{
    // (elements one by one where rows are no whole groups of four; a row's or a column's entries one after the other, up to about 128)
    const double work = entries * (std::max(s.d, 64) / 64.0) * (s.d & 3 ? 1.3 : 1);
    return backward ? 12 + 0.2 * std::min(in_row, 128.0) + (fp32 ? 0.19e-3 : 0.15e-3) * work : 5 + 0.15 * std::min(in_row, 128.0) + 0.06e-3 * work;
}
bool prefer_tiles(const Shape &s, long long nnz, long long tiles, bool backward, bool fp32)
{
    const double problems = (double)s.batch * s.heads, entries = nnz * problems, all = tiles * (problems / s.patterns);
    const double in_row = (double)nnz / s.M, in_block = all / (problems * ((s.M + kTile - 1) / kTile));
    double t;
    if (fp32 && s.d > 64) t = backward ? 85 + 0.32 * all : 38 + 0.06 * std::min(all, 128.0) + 0.6 * in_block + 0.085 * all;
    else if (fp32) t = backward ? 30 + 0.5 * std::min(all, 16.0) + 0.082 * all : 14 + 0.06 * std::min(all, 128.0) + 0.25 * in_block + 0.0225 * all;
    else if (backward) t = 20 + 0.6 * std::min(all, 16.0) + 0.022 * all * (s.d <= 64 ? 1 : 1.6);
    else t = 5 + 1.3 * std::max(in_block / tile_splits(s, tiles).splits, all / 296) + tile_splits(s, tiles).cost;
    if (!fp32 && (s.d & 7)) t += backward ? 10 : 5;   // copies
    return t < row_time(s, entries, in_row, backward, fp32);
}

Call32 call32(const b2sp_attention_problem *p, const Shape &s, char *ws)
{
    Call32 c = {};
    c.s = s;
    c.plan = plan_view(p->plan, plan_layout(s.patterns, s.M, s.K, p->nnz_stride, p->plan_tiles));
    c.tiles = p->plan_tiles;
    c.row_ptr = p->row_ptr; c.col_idx = p->col_idx; c.row_ptr_stride = p->row_ptr_stride; c.nnz_stride = p->nnz_stride;
    c.workspace = ws;
    c.status = reinterpret_cast<int *>(ws + 256);
    return c;
}

template <typename T>
b2sp_status forward(const b2sp_attention_problem *p, const b2sp_heads *Q, const b2sp_heads *K, const b2sp_heads *V, const b2sp_heads *O,
                    float *lse, void *workspace, size_t workspace_bytes, int algo, void *stream)
{
    b2sp_status rc = check_problem(p);
    if (rc != B2SP_OK) return rc;
    if (algo < 0 || algo > B2SP_ALGO_TILE) return B2SP_ERR_INVALID_ARG;
    if ((rc = check_operand(Q, p->M, p->d)) != B2SP_OK || (rc = check_operand(K, p->K, p->d)) != B2SP_OK ||
        (rc = check_operand(V, p->K, p->d)) != B2SP_OK || (rc = check_output(O, p->batch, p->heads, p->M, p->d)) != B2SP_OK)
        return rc;
    if (p->M && !lse) return B2SP_ERR_INVALID_ARG;
    const Shape s = shape(p);
    const RowPlan w = row_plan(s, p->nnz_stride, false, p->plan_tiles, p->plan != nullptr, sizeof(T) == 4);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < w.bytes) return B2SP_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    int &launches = g_launches[0];
    launches = 0;
    if (s.M == 0) return B2SP_OK;
    bool tiles = false;
    if constexpr (sizeof(T) == 2) {
        const View<const T> ops[4] = {view<const T>(Q), view<const T>(K), view<const T>(V), view<const T>(O)};
        const bool can = p->plan && s.K > 0 && tiles_possible(s, ops, 4);
        if (algo == B2SP_ALGO_TILE && !can) return B2SP_ERR_UNSUPPORTED;
        tiles = can && (algo == B2SP_ALGO_TILE || (algo == B2SP_ALGO_AUTO && prefer_tiles(s, p->nnz_stride, p->plan_tiles, false, false)));
        if (tiles) {
            TileCall c = {};
            c.s = s;
            c.plan = plan_view(p->plan, plan_layout(s.patterns, s.M, s.K, p->nnz_stride, p->plan_tiles));
            c.tiles = p->plan_tiles;
            c.row_ptr = p->row_ptr; c.col_idx = p->col_idx; c.row_ptr_stride = p->row_ptr_stride; c.nnz_stride = p->nnz_stride;
            c.q = ops[0]; c.k = ops[1]; c.v = ops[2]; c.out = view<T>(O); c.lse = lse;
            c.workspace = workspace; c.scratch_at = w.ml;
            c.status = reinterpret_cast<int *>(ws + 256);
            g_algo[0] = B2SP_ALGO_TILE;
            return tiles_forward(c, st, &launches);
        }
    } else {
        const bool can = p->plan && tiles32_possible(s, p->plan_tiles, false);
        if (algo == B2SP_ALGO_TILE && !can) return B2SP_ERR_UNSUPPORTED;
        if (can && (algo == B2SP_ALGO_TILE || (algo == B2SP_ALGO_AUTO && prefer_tiles(s, p->nnz_stride, p->plan_tiles, false, true)))) {
            Call32 c = call32(p, s, ws);
            c.q = view<const T>(Q); c.k = view<const T>(K); c.v = view<const T>(V); c.out = view<T>(O); c.lse = lse;
            c.wide_in = fours(c.q, s.d) && fours(c.k, s.d) && fours(c.v, s.d);
            c.wide = fours(c.out, s.d);
            c.scratch_at = w.ml;
            g_algo[0] = B2SP_ALGO_TILE;
            return tiles32_forward(c, st, &launches);
        }
    }
    g_algo[0] = B2SP_ALGO_ROW;
    RowArgs<T> g = {};
    g.s = s;
    g.ptr = p->row_ptr; g.idx = p->col_idx; g.ptr_stride = p->row_ptr_stride; g.idx_stride = p->nnz_stride;
    g.q = view<const T>(Q); g.k = view<const T>(K); g.v = view<const T>(V); g.out1 = view<T>(O);
    g.lse = lse; g.lse_head = s.M; g.lse_row = 1; g.rows = s.M; g.splits = w.splits_m;
    g.status = reinterpret_cast<int *>(ws + 256);
    if (w.splits_m > 1) { g.part = reinterpret_cast<float *>(ws + w.part); g.part_ml = reinterpret_cast<float2 *>(ws + w.ml); }
    const bool wide = fours(g.q, s.d) && fours(g.k, s.d) && fours(g.v, s.d) && fours(g.out1, s.d);
    return launch_rows_v<kForward, T>(wide, g, st, &launches);
}

template <typename T>
b2sp_status backward(const b2sp_attention_problem *p, const b2sp_heads *Q, const b2sp_heads *K, const b2sp_heads *V, const b2sp_heads *O,
                     const float *lse, const b2sp_heads *dO, const b2sp_heads *dQ, const b2sp_heads *dK, const b2sp_heads *dV,
                     void *workspace, size_t workspace_bytes, int algo, void *stream)
{
    b2sp_status rc = check_problem(p);
    if (rc != B2SP_OK) return rc;
    if (algo < 0 || algo > B2SP_ALGO_TILE || !p->plan) return B2SP_ERR_INVALID_ARG;
    if ((rc = check_operand(Q, p->M, p->d)) != B2SP_OK || (rc = check_operand(K, p->K, p->d)) != B2SP_OK ||
        (rc = check_operand(V, p->K, p->d)) != B2SP_OK || (rc = check_operand(O, p->M, p->d)) != B2SP_OK ||
        (rc = check_operand(dO, p->M, p->d)) != B2SP_OK || (rc = check_output(dQ, p->batch, p->heads, p->M, p->d)) != B2SP_OK ||
        (rc = check_output(dK, p->batch, p->kv_heads, p->K, p->d)) != B2SP_OK || (rc = check_output(dV, p->batch, p->kv_heads, p->K, p->d)) != B2SP_OK)
        return rc;
    if (p->M && !lse) return B2SP_ERR_INVALID_ARG;
    const Shape s = shape(p);
    const RowPlan w = row_plan(s, p->nnz_stride, true, p->plan_tiles, true, sizeof(T) == 4);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < w.bytes) return B2SP_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    int &launches = g_launches[1];
    launches = 0;
    const Plan plan = plan_view(p->plan, plan_layout(s.patterns, s.M, s.K, p->nnz_stride, p->plan_tiles));
    bool tiles = false;
    if constexpr (sizeof(T) == 2) {
        const View<const T> ops[8] = {view<const T>(Q), view<const T>(K), view<const T>(V), view<const T>(O), view<const T>(dO), view<const T>(dQ), view<const T>(dK), view<const T>(dV)};
        const bool can = s.M > 0 && s.K > 0 && tiles_possible(s, ops, 8);
        if (algo == B2SP_ALGO_TILE && !can) return B2SP_ERR_UNSUPPORTED;
        tiles = can && (algo == B2SP_ALGO_TILE || (algo == B2SP_ALGO_AUTO && prefer_tiles(s, p->nnz_stride, p->plan_tiles, true, false)));
    } else {
        const bool can = tiles32_possible(s, p->plan_tiles, true);
        if (algo == B2SP_ALGO_TILE && !can) return B2SP_ERR_UNSUPPORTED;
        tiles = can && (algo == B2SP_ALGO_TILE || (algo == B2SP_ALGO_AUTO && prefer_tiles(s, p->nnz_stride, p->plan_tiles, true, true)));
    }
    g_algo[1] = tiles ? B2SP_ALGO_TILE : B2SP_ALGO_ROW;
    float2 *stat = reinterpret_cast<float2 *>(ws + w.stat);
    if constexpr (sizeof(T) == 2) {
        if (tiles) {
            TileCall c = {};
            c.s = s;
            c.plan = plan;
            c.tiles = p->plan_tiles;
            c.row_ptr = p->row_ptr; c.col_idx = p->col_idx; c.row_ptr_stride = p->row_ptr_stride; c.nnz_stride = p->nnz_stride;
            c.q = view<const T>(Q); c.k = view<const T>(K); c.v = view<const T>(V); c.dout = view<const T>(dO);
            c.o = view<const T>(O); c.lse = const_cast<float *>(lse); c.workspace = workspace; c.scratch_at = w.ml;
            c.dq = view<T>(dQ); c.dk = view<T>(dK); c.dv = view<T>(dV);
            c.stat = stat; c.stat_stride = w.stat_rows;
            c.status = reinterpret_cast<int *>(ws + 256);
            return tiles_backward(c, st, &launches);
        }
    }
    if (s.M) {
        const View<const T> o = view<const T>(O), d = view<const T>(dO);
        const long long blocks = ((long long)s.batch * s.heads * w.stat_rows + 7) / 8;
        if (blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
        int *status = reinterpret_cast<int *>(ws + 256);
        if (fours(o, s.d) && fours(d, s.d)) attention_stat_kernel<T, 4><<<(unsigned)blocks, 256, 0, st>>>(s, o, d, lse, w.stat_rows, stat, status);
        else attention_stat_kernel<T, 1><<<(unsigned)blocks, 256, 0, st>>>(s, o, d, lse, w.stat_rows, stat, status);
        ++launches;
        if ((rc = launched()) != B2SP_OK) return rc;
    }
    if constexpr (sizeof(T) == 4) {
        if (tiles) {
            Call32 c = call32(p, s, ws);
            c.q = view<const T>(Q); c.k = view<const T>(K); c.v = view<const T>(V); c.dout = view<const T>(dO);
            c.dq = view<T>(dQ); c.dk = view<T>(dK); c.dv = view<T>(dV);
            c.wide_in = fours(c.q, s.d) && fours(c.k, s.d) && fours(c.v, s.d) && fours(c.dout, s.d);
            c.wide = fours(c.dq, s.d) && fours(c.dk, s.d) && fours(c.dv, s.d);
            c.stat = stat; c.stat_stride = w.stat_rows;
            c.scratch_at = w.ml;
            return tiles32_backward(c, st, &launches);
        }
    }
    RowArgs<T> g = {};
    g.s = s;
    g.q = view<const T>(Q); g.k = view<const T>(K); g.v = view<const T>(V); g.dout = view<const T>(dO);
    g.stat = stat; g.stat_stride = w.stat_rows;
    const bool in = fours(g.q, s.d) && fours(g.k, s.d) && fours(g.v, s.d) && fours(g.dout, s.d);
    g.ptr = p->row_ptr; g.idx = p->col_idx; g.ptr_stride = p->row_ptr_stride; g.idx_stride = p->nnz_stride;
    g.out1 = view<T>(dQ); g.rows = s.M; g.splits = w.splits_m;
    g.part = w.splits_m > 1 ? reinterpret_cast<float *>(ws + w.part) : nullptr;
    if ((rc = launch_rows_v<kGradQ, T>(in && fours(g.out1, s.d), g, st, &launches)) != B2SP_OK) return rc;
    g.ptr = plan.col_ptr; g.idx = plan.row_idx; g.ptr_stride = s.K + 1ll; g.idx_stride = p->nnz_stride;
    g.out1 = view<T>(dK); g.out2 = view<T>(dV); g.rows = s.K; g.splits = w.splits_k;
    g.part = w.parts_kv ? reinterpret_cast<float *>(ws + w.part) : nullptr;
    return launch_rows_v<kGradKV, T>(in && fours(g.out1, s.d) && fours(g.out2, s.d), g, st, &launches);
}

}  // namespace attn
}  // namespace b2sp

using namespace b2sp;
using namespace b2sp::attn;

extern "C" b2sp_status b2sp_attention_count_tiles(int patterns, int M, int K, long long nnz_stride, const int *row_ptr, long long row_ptr_stride,
                                                  const int *col_idx, void *workspace, size_t workspace_bytes, long long *tiles_host, void *stream)
{
    b2sp_status rc = check_pattern(patterns, M, K, nnz_stride, row_ptr, row_ptr_stride, col_idx);
    if (rc != B2SP_OK) return rc;
    if (!tiles_host) return B2SP_ERR_INVALID_ARG;
    const PlanLayout l = plan_layout(patterns, M, K, nnz_stride, 0);
    if (M > kMostPlanRows || l.CB > kMaxColBlocks || (long long)patterns * l.RB > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < 256) return B2SP_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    *tiles_host = 0;
    if (M == 0 || K == 0 || nnz_stride == 0) return B2SP_OK;
    unsigned long long *total = static_cast<unsigned long long *>(workspace);
    if (cudaMemsetAsync(workspace, 0, 256, st) != cudaSuccess) return B2SP_ERR_CUDA;
    plan_mark_kernel<<<patterns * l.RB, 256, l.words * 4, st>>>(Csr{row_ptr, col_idx, row_ptr_stride, nnz_stride, M, K}, l.RB, l.CB, l.words, nullptr, nullptr,
                                                                nullptr, total, reinterpret_cast<int *>(total + 1));
    if ((rc = launched()) != B2SP_OK) return rc;
    unsigned long long n = 0;
    if (cudaMemcpyAsync(&n, total, 8, cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return B2SP_ERR_CUDA;
    if (n > INT_MAX / 2) return B2SP_ERR_UNSUPPORTED;
    *tiles_host = (long long)n;
    return B2SP_OK;
}

extern "C" size_t b2sp_attention_plan_bytes(int patterns, int M, int K, long long nnz_stride, long long tiles)
{
    if (patterns < 1 || M < 0 || K < 0 || nnz_stride < 0 || nnz_stride > INT_MAX || tiles < 0 || tiles > INT_MAX / 2) return 0;
    const PlanLayout l = plan_layout(patterns, M, K, nnz_stride, tiles);
    if (M > kMostPlanRows || l.CB > kMaxColBlocks || (long long)patterns * l.RB > INT_MAX || (long long)patterns * l.CB > INT_MAX) return 0;
    return l.bytes;
}

extern "C" b2sp_status b2sp_attention_prepare(int patterns, int M, int K, long long nnz_stride, const int *row_ptr, long long row_ptr_stride,
                                              const int *col_idx, long long tiles, void *plan, size_t plan_bytes, void *stream)
{
    b2sp_status rc = check_pattern(patterns, M, K, nnz_stride, row_ptr, row_ptr_stride, col_idx);
    if (rc != B2SP_OK) return rc;
    const size_t need = b2sp_attention_plan_bytes(patterns, M, K, nnz_stride, tiles);
    if (!need) return B2SP_ERR_UNSUPPORTED;
    if (!plan || (reinterpret_cast<uintptr_t>(plan) & 255) || plan_bytes < need) return B2SP_ERR_WORKSPACE;
    const PlanLayout l = plan_layout(patterns, M, K, nnz_stride, tiles);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char *b = static_cast<char *>(plan);
    // (everything but the transposed indices begins as zeros: the masks are built by setting bits)
    if (cudaMemsetAsync(plan, 0, l.row_idx, st) != cudaSuccess) return B2SP_ERR_CUDA;
    if (M == 0) return B2SP_OK;
    auto i32 = [&](size_t at) { return reinterpret_cast<int *>(b + at); };
    auto u32 = [&](size_t at) { return reinterpret_cast<unsigned *>(b + at); };
    const Csr s{row_ptr, col_idx, row_ptr_stride, nnz_stride, M, K};
    const int rbs = patterns * l.RB, cbs = patterns * l.CB;
    if (K == 0 || tiles == 0) {   // nothing to list, but row pointers and columns are still checked (all columns may be out of range)
        plan_mark_kernel<<<rbs, 256, l.words * 4, st>>>(s, l.RB, l.CB, l.words, nullptr, nullptr, nullptr, nullptr, i32(0));
        return launched();
    }
    plan_mark_kernel<<<rbs, 256, l.words * 4, st>>>(s, l.RB, l.CB, l.words, u32(l.bitmap), u32(l.rank), i32(l.rb_ptr), nullptr, i32(0));
    plan_scan_kernel<<<1, 1024, 0, st>>>(i32(l.rb_ptr), rbs, 0);
    plan_column_count_kernel<<<(cbs + 127) / 128, 128, 0, st>>>(patterns, l.RB, l.CB, l.words, u32(l.bitmap), i32(l.cb_ptr));
    plan_scan_kernel<<<1, 1024, 0, st>>>(i32(l.cb_ptr), cbs, 0);
    plan_column_list_kernel<<<(cbs + 127) / 128, 128, 0, st>>>(patterns, l.RB, l.CB, l.words, u32(l.bitmap), u32(l.rank), i32(l.rb_ptr), i32(l.cb_ptr),
                                                              tiles, reinterpret_cast<int2 *>(b + l.ctile), i32(l.tile_cb));
    plan_fill_kernel<<<rbs, 512, 0, st>>>(s, l.RB, l.words, u32(l.bitmap), u32(l.rank), i32(l.rb_ptr), tiles, u32(l.masks), i32(0));
    plan_transpose_kernel<<<(unsigned)tiles, kTile, 0, st>>>(patterns, l.CB, K, i32(l.cb_ptr), reinterpret_cast<int2 *>(b + l.ctile),
                                                             reinterpret_cast<uint4 *>(b + l.masks), reinterpret_cast<uint4 *>(b + l.tmasks), i32(l.col_ptr));
    plan_scan_kernel<<<patterns, 1024, 0, st>>>(i32(l.col_ptr), K, K + 1ll);
    plan_rows_kernel<<<cbs, kTile, 0, st>>>(l.CB, K, i32(l.cb_ptr), reinterpret_cast<int2 *>(b + l.ctile), reinterpret_cast<uint4 *>(b + l.tmasks),
                                            i32(l.col_ptr), nnz_stride, i32(l.row_idx));
    return launched();
}

extern "C" b2sp_status b2sp_attention_plan_status(const void *plan, void *stream)
{
    if (!plan) return B2SP_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int h = 0;
    if (cudaMemcpyAsync(&h, plan, sizeof(int), cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return B2SP_ERR_CUDA;
    return h == 0 ? B2SP_OK : B2SP_ERR_BAD_CSR;
}

namespace {
size_t need(const b2sp_attention_problem *p, int backward, bool fp32)
{
    if (check_problem(p) != B2SP_OK || (backward && (p->M > kMostPlanRows || p->K > kMaxColBlocks * kTile))) return 0;   // (backward there is a plan)
    return row_plan(shape(p), p->nnz_stride, backward != 0, p->plan_tiles, p->plan != nullptr || backward, fp32).bytes;
}
}  // namespace
extern "C" size_t b2sp_attention_workspace_bytes(const b2sp_attention_problem *p, int backward) { return need(p, backward, true); }
extern "C" size_t b2sp_attention_workspace_bytes_bf16(const b2sp_attention_problem *p, int backward) { return need(p, backward, false); }

extern "C" b2sp_status b2sp_attention(const b2sp_attention_problem *p, const b2sp_heads *Q, const b2sp_heads *K, const b2sp_heads *V, const b2sp_heads *O,
                                      float *lse, void *workspace, size_t workspace_bytes, int algo, void *stream)
{
    return forward<float>(p, Q, K, V, O, lse, workspace, workspace_bytes, algo, stream);
}
extern "C" b2sp_status b2sp_attention_bf16(const b2sp_attention_problem *p, const b2sp_heads *Q, const b2sp_heads *K, const b2sp_heads *V,
                                           const b2sp_heads *O, float *lse, void *workspace, size_t workspace_bytes, int algo, void *stream)
{
    return forward<Bf16>(p, Q, K, V, O, lse, workspace, workspace_bytes, algo, stream);
}
extern "C" b2sp_status b2sp_attention_backward(const b2sp_attention_problem *p, const b2sp_heads *Q, const b2sp_heads *K, const b2sp_heads *V,
                                               const b2sp_heads *O, const float *lse, const b2sp_heads *dO, const b2sp_heads *dQ, const b2sp_heads *dK,
                                               const b2sp_heads *dV, void *workspace, size_t workspace_bytes, int algo, void *stream)
{
    return backward<float>(p, Q, K, V, O, lse, dO, dQ, dK, dV, workspace, workspace_bytes, algo, stream);
}
extern "C" b2sp_status b2sp_attention_backward_bf16(const b2sp_attention_problem *p, const b2sp_heads *Q, const b2sp_heads *K, const b2sp_heads *V,
                                                    const b2sp_heads *O, const float *lse, const b2sp_heads *dO, const b2sp_heads *dQ,
                                                    const b2sp_heads *dK, const b2sp_heads *dV, void *workspace, size_t workspace_bytes, int algo,
                                                    void *stream)
{
    return backward<Bf16>(p, Q, K, V, O, lse, dO, dQ, dK, dV, workspace, workspace_bytes, algo, stream);
}
extern "C" int b2sp_attention_last_algo(int backward) { return g_algo[backward != 0]; }
extern "C" int b2sp_attention_last_launches(int backward) { return g_launches[backward != 0]; }
