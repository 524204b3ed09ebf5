// Entry points of the 4-bit cache: argument checks and launches.  See include/b2sp.h.
#include <algorithm>
#include <climits>

#include "kv4.cuh"

namespace b2sp {
namespace kv4 {

inline b2sp_status launched() { return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA; }

b2sp_status check_cache(const b2sp_kv4 *c, int heads, int G)
{
    if (!c || c->slots < 0 || c->code_ld < 0 || c->code_stride_head < 0 || c->scale_ld < 0 || c->scale_stride_head < 0) return B2SP_ERR_INVALID_ARG;
    if (c->slots && (!c->codes || !c->scales)) return B2SP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(c->codes) | (uintptr_t)c->code_ld | (uintptr_t)c->code_stride_head) & 15) return B2SP_ERR_INVALID_ARG;
    const int unit = G == 4 ? 4 : G == 2 ? 2 : 1;   // elements that are loaded together
    if (reinterpret_cast<uintptr_t>(c->scales) & (unit == 4 ? 7 : 3)) return B2SP_ERR_INVALID_ARG;
    if (((uintptr_t)c->scale_ld | (uintptr_t)c->scale_stride_head) & (unit - 1)) return B2SP_ERR_INVALID_ARG;
    if (c->slots > 1 && (c->code_ld < 16ll * G || c->scale_ld < G)) return B2SP_ERR_INVALID_ARG;
    return B2SP_OK;
}
// Rows of a cache that is written must not overlap.
b2sp_status check_written(const b2sp_kv4 *c, int heads, int G)
{
    const long long ld[2] = {c->code_ld, c->scale_ld}, sh[2] = {c->code_stride_head, c->scale_stride_head}, row[2] = {16ll * G, G};
    for (int k = 0; k < 2; ++k)
        if (heads > 1 && c->slots > 0 && sh[k] < ld[k] * (c->slots - 1ll) + row[k] && (sh[k] < row[k] || (c->slots > 1 && ld[k] < sh[k] * (heads - 1ll) + row[k])))
            return B2SP_ERR_INVALID_ARG;
    return B2SP_OK;
}
bool below_32_bits(const b2sp_kv4 *c, long long ld, long long sh)
{
    return std::max({c->code_ld, c->code_stride_head, c->scale_ld, c->scale_stride_head, ld, sh}) <= (long long)UINT_MAX;
}
Cache cache(const b2sp_kv4 *c)
{
    return Cache{static_cast<uint8_t *>(c->codes), static_cast<Bf16 *>(c->scales), c->code_ld, c->code_stride_head, c->scale_ld, c->scale_stride_head, c->slots};
}
template <typename T> bool eights(const T *p, long long ld, long long sh, int d)
{
    return ((reinterpret_cast<uintptr_t>(p) & 15) | (uintptr_t)(ld & 7) | (uintptr_t)(sh & 7) | (uintptr_t)(d & 7)) == 0;
}
constexpr int kMost = 0x7fff0000;   // pieces of a launch (indices stay below 2^31)

RowsArgs rows_args(int tokens, int heads, int d, long long ld, long long sh, const int *slots, const b2sp_kv4 *c, unsigned pieces, unsigned first, int *owner)
{
    return RowsArgs{tokens, heads, d, (d + 31) / 32, (unsigned)ld, (unsigned)sh, slots, static_cast<uint8_t *>(c->codes), static_cast<Bf16 *>(c->scales),
                    (unsigned)c->code_ld, (unsigned)c->code_stride_head, (unsigned)c->scale_ld, (unsigned)c->scale_stride_head, c->slots,
                    Div(heads), Div(pieces), first, owner};
}

size_t write_bytes(int tokens, int slots) { return tokens <= kScanTokens ? 0 : (size_t)slots * 4; }

template <typename T>
b2sp_status write(int tokens, int heads, int d, const T *X, long long ld, long long sh, const int *slots, const b2sp_kv4 *c, void *workspace,
                  size_t workspace_bytes, void *stream)
{
    if (tokens < 0 || heads < 1 || d < 1 || ld < 0 || sh < 0) return B2SP_ERR_INVALID_ARG;
    if (tokens && (!X || !slots)) return B2SP_ERR_INVALID_ARG;
    const int G = (d + 31) / 32;
    b2sp_status rc = check_cache(c, heads, G);
    if (rc == B2SP_OK) rc = check_written(c, heads, G);
    if (rc != B2SP_OK) return rc;
    const int each = tokens <= kScanTokens ? 1 : kWritePieces;
    const long long threads = ((long long)tokens + each - 1) / each * heads * G * 4;
    if (d > 32 * 1024 || threads > kMost || !below_32_bits(c, ld, sh)) return B2SP_ERR_UNSUPPORTED;
    const size_t need = write_bytes(tokens, c->slots);
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need)) return B2SP_ERR_WORKSPACE;
    if (c->slots == 0 || tokens == 0) return B2SP_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const RowsArgs a = rows_args(tokens, heads, d, ld, sh, slots, c, 4 * G, 0, static_cast<int *>(workspace));
    const unsigned blocks = (unsigned)((threads + kWriteThreads - 1) / kWriteThreads);
    const bool wide = eights(X, ld, sh, d);
    if (tokens <= kScanTokens) {
        if (wide) kv4_write_kernel<T, 8, true><<<blocks, kWriteThreads, 0, st>>>(X, a);
        else kv4_write_kernel<T, 1, true><<<blocks, kWriteThreads, 0, st>>>(X, a);
    } else {
        const unsigned marks = (tokens + 255) / 256;
        kv4_disown_kernel<<<marks, 256, 0, st>>>(slots, tokens, c->slots, a.owner);
        attn::launch_behind(kv4_own_kernel, marks, 256, st, slots, tokens, c->slots, a.owner);
        if (wide) attn::launch_behind(kv4_write_kernel<T, 8, false>, blocks, kWriteThreads, st, X, a);
        else attn::launch_behind(kv4_write_kernel<T, 1, false>, blocks, kWriteThreads, st, X, a);
    }
    return launched();
}

template <typename T>
b2sp_status read(int tokens, int heads, int d, const int *slots, const b2sp_kv4 *c, T *X, long long ld, long long sh, void *stream)
{
    if (tokens < 0 || heads < 1 || d < 1 || ld < 0 || sh < 0) return B2SP_ERR_INVALID_ARG;
    if (d > 32 * 1024 || (long long)tokens * heads > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    if (tokens && (!X || !slots)) return B2SP_ERR_INVALID_ARG;
    const int G = (d + 31) / 32;
    const b2sp_status rc = check_cache(c, heads, G);
    if (rc != B2SP_OK) return rc;
    if (tokens > 1 && heads > 1 && std::max(ld, sh) < std::min(ld, sh) * ((ld < sh ? tokens : heads) - 1ll) + d) return B2SP_ERR_INVALID_ARG;
    if ((tokens > 1 && ld < d) || (heads > 1 && sh < d)) return B2SP_ERR_INVALID_ARG;
    if (!below_32_bits(c, ld, sh)) return B2SP_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const unsigned pieces = (unsigned)((d + 7) / 8), most = (unsigned)kMost / pieces;
    const bool wide = eights(X, ld, sh, d);
    for (unsigned first = 0, rows = (unsigned)(((long long)tokens + kReadTokens - 1) / kReadTokens * heads); first < rows; first += std::min(most, rows - first)) {
        const RowsArgs a = rows_args(tokens, heads, d, ld, sh, slots, c, pieces, first, nullptr);
        const unsigned blocks = (unsigned)(((unsigned long long)std::min(most, rows - first) * pieces + 255) / 256);
        if (wide) kv4_read_kernel<T, 8><<<blocks, 256, 0, st>>>(a, X);
        else kv4_read_kernel<T, 1><<<blocks, 256, 0, st>>>(a, X);
    }
    return tokens ? launched() : B2SP_OK;
}

struct ServePlan {
    int nb, head_blocks, ctas, share;
    size_t ml, part, bytes;
};
// As many CTAs as run at once (three on an SM), with at least 128 entries each, or one for each token: a CTA takes its tokens one after the other,
// 3 us each however short their lists (122 tokens of up to four slots, 4 heads: 148 us with three CTAs a head, 18 with the call itself with one a token).
ServePlan serve_plan(int M, int heads, int kv_heads, int d, long long nnz)
{
    ServePlan p;
    const int group = heads / kv_heads;
    p.nb = group > 8 ? 2 : 1;
    p.head_blocks = (group + 8 * p.nb - 1) / (8 * p.nb);
    const long long units = (long long)kv_heads * p.head_blocks, most = std::max(1ll, 148ll * 3 / units);
    const long long ctas = std::max(1ll, std::min(most, std::max((nnz + 127) / 128, std::min((long long)M, nnz))));
    p.share = (int)std::max(1ll, (nnz + ctas - 1) / ctas);
    if (p.share >= 128) p.share = (p.share + kSlots - 1) / kSlots * kSlots;
    p.ctas = (int)std::max(1ll, (nnz + p.share - 1) / p.share);
    const long long parts = M > 0 && p.ctas > 1 ? 2ll * p.ctas * heads : 0;
    p.ml = 512;
    p.part = p.ml + attn::up256(parts * 8);
    p.bytes = p.part + attn::up256(parts * attn::part_width(attn::kForward, d) * 4);
    return p;
}

template <int G> void launch(const AttnArgs &a, int nb, unsigned blocks, cudaStream_t st)
{
    if (nb == 2) kv4_attention_kernel<G, 2><<<blocks, attn::kWarps * 32, 0, st>>>(a);
    else kv4_attention_kernel<G, 1><<<blocks, attn::kWarps * 32, 0, st>>>(a);
}

}  // namespace kv4
}  // namespace b2sp

using namespace b2sp;
using namespace b2sp::kv4;

extern "C" size_t b2sp_kv4_write_workspace_bytes(int tokens, int slots)
{
    return tokens < 0 || slots < 0 ? 0 : std::max<size_t>(256, attn::up256(write_bytes(tokens, slots)));
}
extern "C" b2sp_status b2sp_kv4_write(int tokens, int heads, int d, const float *X, long long ld, long long stride_head, const int *slots, const b2sp_kv4 *c,
                                      void *workspace, size_t workspace_bytes, void *stream)
{
    return write<float>(tokens, heads, d, X, ld, stride_head, slots, c, workspace, workspace_bytes, stream);
}
extern "C" b2sp_status b2sp_kv4_write_bf16(int tokens, int heads, int d, const void *X, long long ld, long long stride_head, const int *slots,
                                           const b2sp_kv4 *c, void *workspace, size_t workspace_bytes, void *stream)
{
    return write<Bf16>(tokens, heads, d, static_cast<const Bf16 *>(X), ld, stride_head, slots, c, workspace, workspace_bytes, stream);
}
extern "C" b2sp_status b2sp_kv4_read(int tokens, int heads, int d, const int *slots, const b2sp_kv4 *c, float *X, long long ld, long long stride_head,
                                     void *stream)
{
    return read<float>(tokens, heads, d, slots, c, X, ld, stride_head, stream);
}
extern "C" b2sp_status b2sp_kv4_read_bf16(int tokens, int heads, int d, const int *slots, const b2sp_kv4 *c, void *X, long long ld, long long stride_head,
                                          void *stream)
{
    return read<Bf16>(tokens, heads, d, slots, c, static_cast<Bf16 *>(X), ld, stride_head, stream);
}

static bool serve_args_ok(int M, int heads, int kv_heads, int d, long long nnz)
{
    return M >= 0 && heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0 && d >= 1 && nnz >= 0 && nnz <= INT_MAX;
}

extern "C" size_t b2sp_attention_kv4_workspace_bytes(int M, int heads, int kv_heads, int d, long long nnz)
{
    return serve_args_ok(M, heads, kv_heads, d, nnz) ? serve_plan(M, heads, kv_heads, d, nnz).bytes : 0;
}

extern "C" b2sp_status b2sp_attention_kv4(int M, int heads, int kv_heads, int d, long long nnz, const int *row_ptr, const int *col_idx, const void *Q,
                                          long long ldq, long long stride_head_q, const b2sp_kv4 *keys, const b2sp_kv4 *values, float scale, void *O,
                                          long long ldo, long long stride_head_o, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!serve_args_ok(M, heads, kv_heads, d, nnz) || ldq < 0 || stride_head_q < 0 || !(scale == scale)) return B2SP_ERR_INVALID_ARG;
    if (d > 128) return B2SP_ERR_UNSUPPORTED;
    if (M && (!row_ptr || !Q || !O || !lse || (nnz && !col_idx))) return B2SP_ERR_INVALID_ARG;
    if ((M > 1 && ldo < d) || (heads > 1 && stride_head_o < d)) return B2SP_ERR_INVALID_ARG;
    if (M > 1 && heads > 1 && std::max(ldo, stride_head_o) < std::min(ldo, stride_head_o) * ((ldo < stride_head_o ? M : heads) - 1ll) + d) return B2SP_ERR_INVALID_ARG;
    const int G = (d + 31) / 32;
    b2sp_status rc = check_cache(keys, kv_heads, G);
    if (rc == B2SP_OK) rc = check_cache(values, kv_heads, G);
    if (rc != B2SP_OK) return rc;
    if (keys->code_ld > INT_MAX || values->code_ld > INT_MAX || keys->scale_ld > INT_MAX || values->scale_ld > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    const ServePlan p = serve_plan(M, heads, kv_heads, d, nnz);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < p.bytes) return B2SP_ERR_WORKSPACE;
    if (M == 0) return B2SP_OK;
    const long long blocks = (long long)kv_heads * p.head_blocks * p.ctas, joins = (long long)M * heads;
    if (blocks > INT_MAX || joins > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    AttnArgs a = {};
    a.M = M; a.heads = heads; a.kv_heads = kv_heads; a.d = d; a.head_blocks = p.head_blocks; a.ctas = p.ctas; a.share = p.share; a.nnz = nnz;
    a.row_ptr = row_ptr; a.col_idx = col_idx;
    a.q = static_cast<const Bf16 *>(Q); a.q_ld = ldq; a.q_sh = stride_head_q;
    a.q_wide = eights(a.q, ldq, stride_head_q, d);
    a.k = cache(keys); a.v = cache(values); a.scale = scale;
    a.out = attn::View<Bf16>{static_cast<Bf16 *>(O), ldo, stride_head_o, 0};
    a.lse = lse;
    a.part = reinterpret_cast<float *>(ws + p.part);
    a.part_ml = reinterpret_cast<float2 *>(ws + p.ml);
    if (nnz) {
        switch (G) {
            case 1: launch<1>(a, p.nb, (unsigned)blocks, st); break;
            case 2: launch<2>(a, p.nb, (unsigned)blocks, st); break;
            case 3: launch<3>(a, p.nb, (unsigned)blocks, st); break;
            default: launch<4>(a, p.nb, (unsigned)blocks, st); break;
        }
        attn::launch_behind(kv4_join_kernel, (unsigned)joins, kJoinWarps * 32, st, a);
    } else {
        kv4_join_kernel<<<(unsigned)joins, kJoinWarps * 32, 0, st>>>(a);
    }
    return launched();
}
