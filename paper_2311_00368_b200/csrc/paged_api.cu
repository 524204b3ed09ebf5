// Entry points of the cache in pages: argument checks and launches.  See include/b2sp.h.
#include <algorithm>
#include <atomic>
#include <climits>

#include "overlap.h"
#include "paged_attention.cuh"

namespace b2sp {
namespace paged {

inline b2sp_status launched() { return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA; }
constexpr int kSMs = 148, kMostTokens = 1 << 30;
constexpr size_t kMostShared = 227 * 1024;   // of a CTA

// More shared memory than a launch gets unasked (48 KB with what the kernel has of its own): asked for once on each device.
template <auto Kernel> bool allow_shared(size_t bytes)
{
    if (bytes <= 40 * 1024) return true;
    static std::atomic<size_t> allowed[64];
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return false;
    std::atomic<size_t> *mine = device < 64 ? allowed + device : nullptr;
    if (mine && mine->load() >= bytes) return true;
    // as much as the kernel can have, whatever this call needs: so no call takes away what another has asked for
    cudaFuncAttributes has;
    if (cudaFuncGetAttributes(&has, Kernel) != cudaSuccess) return false;
    const size_t most = kMostShared - has.sharedSizeBytes;
    if (bytes > most || cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most) != cudaSuccess) return false;
    if (mine) mine->store(most);
    return true;
}
// A launch that may begin before the one ahead of it has ended (the kernels wait for that themselves).
template <auto Kernel, typename... Args> bool launch_early(dim3 blocks, unsigned threads, size_t shared, cudaStream_t st, const Args &...args)
{
    if (!allow_shared<Kernel>(shared)) { cudaGetLastError(); return false; }   // (an error that stays is the next call's)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, Kernel, args...) == cudaSuccess) return true;
    cudaGetLastError();
    return false;
}

b2sp_status check_tables(const b2sp_page_tables *t, int page)
{
    if (!t || t->requests < 0 || t->width < 0 || t->ld < 0 || page < 1) return B2SP_ERR_INVALID_ARG;
    if (t->requests && t->width && !t->entries) return B2SP_ERR_INVALID_ARG;
    return B2SP_OK;
}
Tables tables(const b2sp_page_tables *t) { return Tables{t->entries, t->ld, t->requests, t->width}; }

// rows: rows of a page (a cache) or 1 (means: ld is not looked at).
template <typename T> b2sp_status check_pages(const b2sp_pages *c, int heads, int d, int rows)
{
    if (!c || c->pages < 0 || c->page < 1 || c->ld < 0 || c->stride_head < 0 || c->stride_page < 0) return B2SP_ERR_INVALID_ARG;
    if (c->pages && !c->data) return B2SP_ERR_INVALID_ARG;
    const uintptr_t strides = (rows > 1 ? (uintptr_t)c->ld : 0) | (uintptr_t)c->stride_head | (uintptr_t)c->stride_page;
    if ((reinterpret_cast<uintptr_t>(c->data) | strides * sizeof(T)) & 15) return B2SP_ERR_INVALID_ARG;
    if (rows > 1 && c->ld < d) return B2SP_ERR_INVALID_ARG;
    return B2SP_OK;
}
// What is written must not overlap: sorted by stride, each dimension's stride is at least the extent of those within it.
bool apart(int d, std::initializer_list<std::pair<long long, long long>> dims)   // (size, stride)
{
    std::pair<long long, long long> v[3];
    int n = 0;
    for (const auto &x : dims)
        if (x.first > 1) v[n++] = x;
    std::sort(v, v + n, [](const auto &x, const auto &y) { return x.second < y.second; });
    __int128 extent = d;
    for (int i = 0; i < n; ++i) {
        if (v[i].second < extent) return false;
        extent += (__int128)(v[i].first - 1) * v[i].second;
    }
    return true;
}
template <typename T> Pages<T> pages(const b2sp_pages *c) { return Pages<T>{static_cast<T *>(c->data), c->ld, c->stride_head, c->stride_page, c->pages}; }
bool same_slots(const b2sp_pages *a, const b2sp_pages *b) { return a->pages == b->pages && a->page == b->page; }
long long bytes_of(long long stride, size_t wide) { return std::min(stride, 1ll << 58) * (long long)wide; }   // (no two rows lie further apart)
template <typename T> Spread spread(const b2sp_pages *c, int heads, int d, int rows)   // rows: of a page, 1 for means
{
    return Spread(c->data, d * sizeof(T), {{c->pages, bytes_of(c->stride_page, sizeof(T))}, {heads, bytes_of(c->stride_head, sizeof(T))}, {rows, bytes_of(c->ld, sizeof(T))}});
}
template <typename T> Spread spread(const T *x, int tokens, long long ld, int heads, long long sh, int d)
{
    return Spread(x, d * sizeof(T), {{tokens, bytes_of(ld, sizeof(T))}, {heads, bytes_of(sh, sizeof(T))}});
}
Spread spread(const b2sp_page_tables *t) { return Spread(t->entries, t->width * 4ll, {{t->requests, bytes_of(t->ld, 4)}}); }
Spread ints(const int *x, long long n) { return Spread(x, std::min(n, 1ll << 58) * 4); }
// Whether an output lies in one of the inputs or in another output: CTAs read the ones while others write.
bool mixed(std::initializer_list<Spread> out, std::initializer_list<Spread> in)
{
    for (auto x = out.begin(); x != out.end(); ++x) {
        for (const Spread &y : in)
            if (share(*x, y)) return true;
        for (auto y = x + 1; y != out.end(); ++y)
            if (share(*x, *y)) return true;
    }
    return false;
}

template <typename T> bool fits(const void *x, long long ld, long long sh, size_t bytes)   // rows begin on multiples of `bytes`
{
    return ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(ld * (long long)sizeof(T)) | (uintptr_t)(sh * (long long)sizeof(T))) & (bytes - 1)) == 0;
}

template <typename T>
b2sp_status write(int tokens, int heads, int d, const T *K, long long ldk, long long shk, const T *V, long long ldv, long long shv, const int *row_ptr,
                  const int *lengths, const b2sp_page_tables *t, const b2sp_pages *kp, const b2sp_pages *vp, const b2sp_pages *means, void *stream)
{
    if (tokens < 0 || heads < 1 || d < 1 || ldk < 0 || shk < 0 || ldv < 0 || shv < 0) return B2SP_ERR_INVALID_ARG;
    b2sp_status rc = check_pages<T>(kp, heads, d, 2);
    if (rc == B2SP_OK) rc = check_pages<T>(vp, heads, d, 2);
    if (rc == B2SP_OK && means) rc = check_pages<T>(means, heads, d, 1);
    if (rc == B2SP_OK) rc = check_tables(t, kp->page);
    if (rc != B2SP_OK) return rc;
    if (t->requests > kMostRequests || d > 1024) return B2SP_ERR_UNSUPPORTED;
    if (!same_slots(kp, vp) || (means && means->pages != kp->pages)) return B2SP_ERR_INVALID_ARG;
    for (const b2sp_pages *c : {kp, vp})
        if (!apart(d, {{c->pages, c->stride_page}, {heads, c->stride_head}, {c->page, c->ld}})) return B2SP_ERR_INVALID_ARG;
    if (means && !apart(d, {{means->pages, means->stride_page}, {heads, means->stride_head}})) return B2SP_ERR_INVALID_ARG;
    if (t->requests && (!row_ptr || !lengths)) return B2SP_ERR_INVALID_ARG;
    if (tokens && (!K || !V)) return B2SP_ERR_INVALID_ARG;
    const int R = t->requests;
    if (mixed({spread<T>(kp, heads, d, kp->page), spread<T>(vp, heads, d, kp->page), means ? spread<T>(means, heads, d, 1) : Spread(nullptr, 0)},
              {ints(row_ptr, R + 1), ints(lengths, R), spread(t)}))
        return B2SP_ERR_INVALID_ARG;
    if (tokens == 0 || t->requests == 0 || kp->pages == 0) return B2SP_OK;
    WriteArgs<T> a = {};
    a.t = tables(t);
    a.k = K; a.v = V; a.k_ld = ldk; a.k_sh = shk; a.v_ld = ldv; a.v_sh = shv;
    a.heads = heads; a.d = d; a.page = kp->page; a.tokens = tokens; a.row_ptr = row_ptr; a.lengths = lengths;
    a.kp = pages<T>(kp); a.vp = pages<T>(vp);
    if (means) a.means = pages<T>(means);
    // as many pages as the tokens can touch: at most two that are not full for each request that has any
    const long long units = (tokens / kp->page + 2ll * std::min(t->requests, tokens)) * heads;
    const unsigned blocks = (unsigned)std::min(units, (long long)kWriteCTAs * kSMs);
    const size_t shared = (t->requests + 1) * sizeof(int);
    return launch_early<paged_write_kernel<T>>(blocks, kWriteThreads, shared, static_cast<cudaStream_t>(stream), a) ? launched() : B2SP_ERR_CUDA;
}

bool token_args_ok(int M, int heads, int kv_heads, int d) { return M >= 0 && heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0 && d >= 1; }

// A workspace begins with what b2sp_device_status reads, as those of the other calls do.
constexpr size_t kHead = 512, kStatus = 256;
size_t select_bytes(int M, int kv_heads, int width) { return kHead + attn::up256((size_t)M * kv_heads * width * sizeof(float2)); }

template <typename T>
b2sp_status select(int M, int heads, int kv_heads, int d, const T *Q, long long ldq, long long shq, const b2sp_pages *means, const b2sp_page_tables *t,
                   const int *rows, const int *seen, int keep, int first, int last, int *lists, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!token_args_ok(M, heads, kv_heads, d) || ldq < 0 || shq < 0 || keep < 1 || first < 0 || last < 0 || first > keep - last) return B2SP_ERR_INVALID_ARG;
    b2sp_status rc = check_pages<T>(means, kv_heads, d, 1);
    if (rc == B2SP_OK) rc = check_tables(t, means->page);
    if (rc != B2SP_OK) return rc;
    if (M && (!Q || !seen || !lists)) return B2SP_ERR_INVALID_ARG;
    if (d > 256 || M > kMostTokens || std::max(means->stride_head, means->stride_page) > (long long)(UINT_MAX / sizeof(T))) return B2SP_ERR_UNSUPPORTED;
    const long long blocks = (long long)M * kv_heads * (((long long)t->width + 7) / 8), ctas = (long long)M * kv_heads;   // blocks: of eight pages at least
    if (ctas > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < select_bytes(M, kv_heads, t->width)) return B2SP_ERR_WORKSPACE;
    if (M == 0) return B2SP_OK;
    if (mixed({ints(lists, ctas * keep)}, {ints(seen, M), ints(rows, M), spread(t), spread(Q, M, ldq, heads, shq, d), spread<T>(means, kv_heads, d, 1)}))
        return B2SP_ERR_INVALID_ARG;
    SelectArgs<T> a = {};
    a.t = tables(t);
    a.tok = Tokens{rows, seen};
    a.q = Q; a.q_ld = ldq; a.q_sh = shq;
    a.M = M; a.heads = heads; a.kv_heads = kv_heads; a.d = d; a.page = means->page; a.keep = keep; a.first = first; a.last = last;
    a.means = pages<T>(means);
    a.status = reinterpret_cast<int *>(static_cast<char *>(workspace) + kStatus);
    a.scores = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + kHead);
    a.lists = lists;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    a.q_wide = fits<T>(Q, ldq, shq, 16);
    const bool scored = t->width > keep;   // else no token sees more pages than a list holds
    if (scored) {
        constexpr int N = 16 / sizeof(T);
        const unsigned grid = (unsigned)std::min((blocks + kScoreThreads / 32 - 1) / (kScoreThreads / 32), (long long)kSMs * (d <= 32 * N ? kScoreCTAs : kScoreCTAs / 2));
        constexpr size_t room = kScoreThreads * (kScoreAhead + 1) * 8 * 16;   // eight loads of 16 bytes of a lane
        bool ok = false;
        if (d <= 8 * N) ok = launch_early<paged_score_kernel<T, 8, 1>>(grid, kScoreThreads, room, st, a);
        else if (d <= 16 * N) ok = launch_early<paged_score_kernel<T, 16, 1>>(grid, kScoreThreads, room, st, a);
        else if (d <= 32 * N) ok = launch_early<paged_score_kernel<T, 32, 1>>(grid, kScoreThreads, room, st, a);
        else if constexpr (sizeof(T) == 4) ok = launch_early<paged_score_kernel<T, 32, 2>>(grid, kScoreThreads, 2 * room, st, a);
        if (!ok) return B2SP_ERR_CUDA;
    }
    // Eight keys a lane where that can be: more of them are more code, which runs once (one warp's 64: 69.7 instead of 50.8 us for 64 tokens that see up to 2048
    // pages, 8 key heads; its 32: 20.6 instead of 19.2 for up to 512).  One warp where that is enough (four: 24.4 instead of 20.0 us for 256 tokens, up to 125).
    const bool ok = t->width <= 256    ? launch_early<paged_select_kernel<T, 1, 8>>((unsigned)((ctas + 3) / 4), 128, 0, st, a, scored)
                    : t->width <= 1024 ? launch_early<paged_select_kernel<T, 4, 8>>((unsigned)ctas, 128, 0, st, a, scored)
                    : t->width <= 2048 ? launch_early<paged_select_kernel<T, 8, 8>>((unsigned)ctas, 256, 0, st, a, scored)
                                       : launch_early<paged_select_kernel<T, 8, 64>>((unsigned)ctas, 256, 0, st, a, scored);
    if (!ok) return B2SP_ERR_CUDA;
    return launched();
}

// Warps and workspace of an attention call.
struct AttnPlan {
    int queries, blocks, warps;   // queries: of a unit; blocks: units of a token and key head; warps: at most
    size_t ml, part, bytes;
};
// together: tokens of a request that are likely to be neighbours (1 with lists or without `rows`).
template <typename T> AttnPlan attention_plan(int heads, int kv_heads, int d, long long together)
{
    AttnPlan p;
    const int group = heads / kv_heads, w = d <= 64 ? 64 : d <= 128 ? 128 : 256;
    p.queries = sizeof(T) == 2 ? (group * together > 8 ? 16 : 8) : group * together > 4 ? 8 : 4;
    p.blocks = (group + p.queries - 1) / p.queries;
    p.warps = kSMs * kAttnWarps * (w == 64 ? Form<T, 64>::CTAS : w == 128 ? Form<T, 128>::CTAS : Form<T, 256>::CTAS);
    const size_t parts = 2ull * p.warps * p.queries;
    p.ml = kHead + attn::up256(p.warps * sizeof(int4));
    p.part = p.ml + attn::up256(parts * sizeof(float2));
    p.bytes = p.part + attn::up256(parts * w * sizeof(float));
    return p;
}

size_t attention_bytes(int heads, int kv_heads, int d)   // for either type and any tokens
{
    return std::max(attention_plan<float>(heads, kv_heads, d, INT_MAX).bytes, attention_plan<Bf16>(heads, kv_heads, d, INT_MAX).bytes);
}

template <typename T, int W, int Q> b2sp_status launch_attention(AttnArgs<T> &a, const AttnPlan &p, long long most_tiles, cudaStream_t st)
{
    using F = Form<T, W, Q>;
    static_assert(F::CTAS == Form<T, W>::CTAS, "");
    const long long units = (long long)a.M * a.kv_heads * a.blocks, most_cost = most_tiles + units * kUnitCost;
    // no more CTAs than have a share, if every token sees all that it can
    const unsigned ctas = (unsigned)std::min((long long)kSMs * F::CTAS, (most_cost + kLeastCost * kAttnWarps - 1) / (kLeastCost * kAttnWarps));
    if (most_cost / (ctas * kAttnWarps) >= 1 << 30) return B2SP_ERR_UNSUPPORTED;   // (a warp counts its share in 32 bits)
    a.by_unit = units <= ctas * (long long)kAttnWarps;
    const bool ok = a.page % F::ROWS == 0 ? launch_early<paged_attention_kernel<T, W, Q, true>>(ctas, kAttnWarps * 32, F::SHARED, st, a)
                                          : launch_early<paged_attention_kernel<T, W, Q, false>>(ctas, kAttnWarps * 32, F::SHARED, st, a);
    if (!ok) return B2SP_ERR_CUDA;
    // Few units have many parts each: sixteen warps for a query, else one.
    const unsigned joins = a.by_unit ? (unsigned)units : ctas * kAttnWarps, queries = std::min(a.pack * a.group, p.queries);
    const bool joined = units * 16 <= ctas * kAttnWarps
                            ? launch_early<paged_join_kernel<T, W, 16>>(dim3(joins, queries), 512, 0, st, a, p.queries)
                            : launch_early<paged_join_kernel<T, W, 1>>(dim3(joins, (queries + 7) / 8), 256, 0, st, a, p.queries);
    return joined ? launched() : B2SP_ERR_CUDA;
}

template <typename T>
b2sp_status attention(int M, int heads, int kv_heads, int d, const T *Q, long long ldq, long long shq, const b2sp_pages *kp, const b2sp_pages *vp,
                      const b2sp_page_tables *t, const int *rows, const int *seen, const int *lists, int keep, float scale, T *O, long long ldo,
                      long long sho, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!token_args_ok(M, heads, kv_heads, d) || ldq < 0 || shq < 0 || ldo < 0 || sho < 0 || !(scale == scale) || (lists && keep < 1)) return B2SP_ERR_INVALID_ARG;
    b2sp_status rc = check_pages<T>(kp, kv_heads, d, 2);
    if (rc == B2SP_OK) rc = check_pages<T>(vp, kv_heads, d, 2);
    if (rc == B2SP_OK) rc = check_tables(t, kp->page);
    if (rc != B2SP_OK) return rc;
    if (!same_slots(kp, vp)) return B2SP_ERR_INVALID_ARG;
    if (M && (!Q || !O || !lse || !seen)) return B2SP_ERR_INVALID_ARG;
    if (!apart(d, {{M, ldo}, {heads, sho}})) return B2SP_ERR_INVALID_ARG;
    if (d > 256 || M > kMostTokens || (lists && (long long)keep * kp->page > INT_MAX) || (long long)M * heads > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    constexpr long long most_stride = UINT_MAX / sizeof(T);
    for (const b2sp_pages *c : {kp, vp})
        if (std::max({c->ld, c->stride_head, c->stride_page, ldq, shq, ldo, sho, t->ld}) > most_stride) return B2SP_ERR_UNSUPPORTED;
    const AttnPlan p = attention_plan<T>(heads, kv_heads, d, rows && !lists && t->requests ? M / t->requests : 1);
    if ((long long)M * kv_heads * p.blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < attention_bytes(heads, kv_heads, d)) return B2SP_ERR_WORKSPACE;
    if (M == 0) return B2SP_OK;
    const Spread q = spread(Q, M, ldq, heads, shq, d), o = spread(O, M, ldo, heads, sho, d);
    if (mixed({o, Spread(lse, (long long)M * heads * 4)}, {ints(seen, M), ints(rows, M), spread(t), ints(lists, (long long)M * kv_heads * keep),
                                                           spread<T>(kp, kv_heads, d, kp->page), spread<T>(vp, kv_heads, d, kp->page)}))
        return B2SP_ERR_INVALID_ARG;
    if (!(q == o) && mixed({o, Spread(lse, (long long)M * heads * 4)}, {q})) return B2SP_ERR_INVALID_ARG;
    AttnArgs<T> a = {};
    a.t = tables(t);
    a.tok = Tokens{rows, seen};
    a.q = Q; a.q_ld = (unsigned)ldq; a.q_sh = (unsigned)shq;
    a.M = M; a.heads = heads; a.kv_heads = kv_heads; a.d = d; a.page = kp->page;
    const auto side = [](const b2sp_pages *c) {
        return Side{static_cast<const char *>(c->data), (unsigned)(c->ld * sizeof(T)), (unsigned)(c->stride_head * sizeof(T)), (unsigned)(c->stride_page * sizeof(T))};
    };
    a.k = side(kp); a.v = side(vp); a.pages = kp->pages;
    a.lists = lists; a.keep = lists ? keep : 0; a.scale = scale;
    a.out = O; a.out_ld = (unsigned)ldo; a.out_sh = (unsigned)sho; a.lse = lse;
    a.group = heads / kv_heads; a.blocks = p.blocks; a.by_page = Div(a.page);
    a.pack = 1;
    if (rows && !lists)
        while (a.pack * 2 * a.group <= p.queries) a.pack *= 2;
    a.by_blocks = Div(p.blocks);
    a.by_heads = Div(a.pack > 1 ? a.group : p.queries);
    a.pairs = fits<T>(Q, ldq, shq, 4) && fits<T>(O, ldo, sho, 4) && d % 2 == 0;
    a.fours = fits<T>(Q, ldq, shq, 16) && (sizeof(T) == 2 || d % 4 == 0);
    char *ws = static_cast<char *>(workspace);
    a.status = reinterpret_cast<int *>(ws + kStatus);
    a.joins = reinterpret_cast<int4 *>(ws + kHead);
    a.part_ml = reinterpret_cast<float2 *>(ws + p.ml);
    a.part = reinterpret_cast<float *>(ws + p.part);
    const long long most_rows = lists ? (long long)keep * a.page : (long long)t->width * a.page, units = (long long)M * kv_heads * p.blocks;
    const __int128 tiles = (__int128)units * std::max(1ll, (most_rows + 7) / 8);
    const long long most = (long long)std::min<__int128>(tiles, 1ll << 40);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int w = d <= 64 ? 64 : d <= 128 ? 128 : 256;
    constexpr int MOST = sizeof(T) == 2 ? 16 : 8;
    if (p.queries == MOST) return w == 64 ? launch_attention<T, 64, MOST>(a, p, most, st) : w == 128 ? launch_attention<T, 128, MOST>(a, p, most, st) : launch_attention<T, 256, MOST>(a, p, most, st);
    return w == 64 ? launch_attention<T, 64, MOST / 2>(a, p, most, st) : w == 128 ? launch_attention<T, 128, MOST / 2>(a, p, most, st) : launch_attention<T, 256, MOST / 2>(a, p, most, st);
}

}  // namespace paged
}  // namespace b2sp

using namespace b2sp;
using namespace b2sp::paged;

extern "C" b2sp_status b2sp_paged_tables(const b2sp_page_tables *t, int pages, int page, const int *lengths, const int *added, int *free_pages,
                                         int free_room, const int *free_count, int tokens, int *lengths_out, int *row_ptr, int *rows, int *seen,
                                         int *slots, int *counts, void *stream)
{
    b2sp_status rc = check_tables(t, page);
    if (rc != B2SP_OK) return rc;
    const int R = t->requests;
    if (pages < 0 || free_room < 0 || tokens < 0 || (R > 1 && t->ld < t->width)) return B2SP_ERR_INVALID_ARG;
    if (!row_ptr || !counts || !free_count || (R && (!lengths || !added || !lengths_out)) || (free_room && !free_pages)) return B2SP_ERR_INVALID_ARG;
    if (tokens && (!rows || !seen || !slots)) return B2SP_ERR_INVALID_ARG;
    if (R > kMostRequests || (long long)pages * page > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    if (mixed({ints(lengths_out, R), ints(row_ptr, R + 1), ints(rows, tokens), ints(seen, tokens), ints(slots, tokens), ints(counts, 4), ints(free_pages, free_room),
               spread(t)}, {ints(lengths, R), ints(added, R), ints(free_count, 1)}))
        return B2SP_ERR_INVALID_ARG;
    const size_t shared = 3 * (R + 1) * sizeof(int);
    TablesArgs a = {};
    a.t = tables(t);
    a.page = page; a.pages = pages; a.tokens = tokens; a.free_room = free_room;
    a.lengths = lengths; a.added = added; a.free_count = free_count; a.free_pages = free_pages;
    a.lengths_out = lengths_out; a.row_ptr = row_ptr; a.rows = rows; a.seen = seen; a.slots = slots; a.counts = counts;
    const unsigned blocks = (unsigned)std::min(std::max(((long long)std::max(tokens, R) + kThreads - 1) / kThreads, 1ll), 2ll * kSMs);
    return launch_early<paged_tables_kernel>(blocks, kThreads, shared, static_cast<cudaStream_t>(stream), a) ? launched() : B2SP_ERR_CUDA;
}

extern "C" b2sp_status b2sp_paged_lists(int M, const b2sp_page_tables *t, int pages, int page, const int *rows, const int *seen, long long entries,
                                        int *row_ptr, int *col_idx, void *stream)
{
    b2sp_status rc = check_tables(t, page);
    if (rc != B2SP_OK) return rc;
    if (M < 0 || pages < 0 || entries < 0 || !row_ptr || (M && !seen) || (entries && !col_idx)) return B2SP_ERR_INVALID_ARG;
    if (entries > INT_MAX || (long long)pages * page > INT_MAX || M > kMostTokens) return B2SP_ERR_UNSUPPORTED;
    if (mixed({ints(row_ptr, M + 1ll), ints(col_idx, entries)}, {ints(seen, M), ints(rows, M), spread(t)})) return B2SP_ERR_INVALID_ARG;
    ListsArgs a = {};
    a.t = tables(t);
    a.tok = Tokens{rows, seen};
    a.M = M; a.page = page; a.pages = pages; a.entries = entries; a.row_ptr = row_ptr; a.col_idx = col_idx; a.by_page = Div(page);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const unsigned blocks = (unsigned)std::min(std::max((entries + 4 * kThreads - 1) / (4 * kThreads), 1ll), 8ll * kSMs);
    bool ok;
    if (M <= kListTokens) {
        ok = launch_early<paged_list_kernel<true>>(blocks, kThreads, (M + 1) * sizeof(int), st, a);
    } else {
        ok = launch_early<paged_list_ends_kernel>(1, kScanThreads, 0, st, a);
        if (ok && entries) ok = launch_early<paged_list_kernel<false>>(blocks, kThreads, 0, st, a);
    }
    if (!ok) return B2SP_ERR_CUDA;
    return launched();
}

extern "C" b2sp_status b2sp_paged_write(int tokens, int heads, int d, const float *K, long long ldk, long long shk, const float *V, long long ldv,
                                        long long shv, const int *row_ptr, const int *lengths, const b2sp_page_tables *t, const b2sp_pages *kp,
                                        const b2sp_pages *vp, const b2sp_pages *means, void *stream)
{
    return write<float>(tokens, heads, d, K, ldk, shk, V, ldv, shv, row_ptr, lengths, t, kp, vp, means, stream);
}
extern "C" b2sp_status b2sp_paged_write_bf16(int tokens, int heads, int d, const void *K, long long ldk, long long shk, const void *V, long long ldv,
                                             long long shv, const int *row_ptr, const int *lengths, const b2sp_page_tables *t, const b2sp_pages *kp,
                                             const b2sp_pages *vp, const b2sp_pages *means, void *stream)
{
    return write<Bf16>(tokens, heads, d, static_cast<const Bf16 *>(K), ldk, shk, static_cast<const Bf16 *>(V), ldv, shv, row_ptr, lengths, t, kp, vp,
                       means, stream);
}

extern "C" size_t b2sp_paged_select_workspace_bytes(int M, int kv_heads, int width)
{
    return M < 0 || kv_heads < 1 || width < 0 ? 0 : select_bytes(M, kv_heads, width);
}
extern "C" b2sp_status b2sp_paged_select(int M, int heads, int kv_heads, int d, const float *Q, long long ldq, long long shq, const b2sp_pages *means,
                                         const b2sp_page_tables *t, const int *rows, const int *seen, int keep, int first, int last, int *lists,
                                         void *workspace, size_t workspace_bytes, void *stream)
{
    return paged::select<float>(M, heads, kv_heads, d, Q, ldq, shq, means, t, rows, seen, keep, first, last, lists, workspace, workspace_bytes, stream);
}
extern "C" b2sp_status b2sp_paged_select_bf16(int M, int heads, int kv_heads, int d, const void *Q, long long ldq, long long shq, const b2sp_pages *means,
                                              const b2sp_page_tables *t, const int *rows, const int *seen, int keep, int first, int last, int *lists,
                                              void *workspace, size_t workspace_bytes, void *stream)
{
    return paged::select<Bf16>(M, heads, kv_heads, d, static_cast<const Bf16 *>(Q), ldq, shq, means, t, rows, seen, keep, first, last, lists, workspace,
                               workspace_bytes, stream);
}

extern "C" size_t b2sp_attention_paged_workspace_bytes(int M, int heads, int kv_heads, int d)
{
    if (!token_args_ok(M, heads, kv_heads, d) || d > 256) return 0;
    return attention_bytes(heads, kv_heads, d);
}
extern "C" b2sp_status b2sp_attention_paged(int M, int heads, int kv_heads, int d, const float *Q, long long ldq, long long shq, const b2sp_pages *kp,
                                            const b2sp_pages *vp, const b2sp_page_tables *t, const int *rows, const int *seen, const int *lists, int keep,
                                            float scale, float *O, long long ldo, long long sho, float *lse, void *workspace, size_t workspace_bytes,
                                            void *stream)
{
    return attention<float>(M, heads, kv_heads, d, Q, ldq, shq, kp, vp, t, rows, seen, lists, keep, scale, O, ldo, sho, lse, workspace, workspace_bytes,
                            stream);
}
extern "C" b2sp_status b2sp_attention_paged_bf16(int M, int heads, int kv_heads, int d, const void *Q, long long ldq, long long shq, const b2sp_pages *kp,
                                                 const b2sp_pages *vp, const b2sp_page_tables *t, const int *rows, const int *seen, const int *lists,
                                                 int keep, float scale, void *O, long long ldo, long long sho, float *lse, void *workspace,
                                                 size_t workspace_bytes, void *stream)
{
    return attention<Bf16>(M, heads, kv_heads, d, static_cast<const Bf16 *>(Q), ldq, shq, kp, vp, t, rows, seen, lists, keep, scale,
                           static_cast<Bf16 *>(O), ldo, sho, lse, workspace, workspace_bytes, stream);
}
