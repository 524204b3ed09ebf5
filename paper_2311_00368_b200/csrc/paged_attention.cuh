// Attention of new tokens over a cache in pages.
//
//   s_j = scale q . k_j;  O = sum_j exp(s_j - m) v_j / l,  l = sum_j exp(s_j - m),  lse = m + log l
//
// over the positions j that a token sees, or those of them in the pages that its list names.  Every row of the cache is read once for the heads that
// share it and used 2 to 16 times, so HBM bounds the work and everything else has to keep out of its way.
//
// A unit is a key head and up to 8 (16) queries that look at it: the heads that share it, of one token or of neighbouring tokens of one request; its rows
// come in tiles of 16 (8).  All units' tiles in a line are dealt to the warps in equal shares: a warp takes its share by itself, with a ring of tiles of its
// own in shared memory that asynchronous copies fill two tiles ahead, and waits for no other warp.  It knows its share from prefix sums over the tokens, so
// lengths stay on the device and a long row is spread over the GPU as well as many short ones.  Units that end up in several shares leave their sums in
// the workspace, and a second kernel joins them in order.
// Rows that are not there (behind what is seen, of missing pages) are filled with zeros by the copies instead of read: what memory holds there does not
// enter.
#pragma once
#include "paged.cuh"

namespace b2sp {
namespace paged {

constexpr int kAttnWarps = 4, kStages = 3;   // warps of a CTA; tiles of a warp in shared memory
// A unit costs its tiles and, before the first one, a chain of latencies (lengths, table, rows), as long as about four tiles take: without it warps whose
// shares were many short units took twice as long as the others.  Shares are of at least kLeastCost.
constexpr int kUnitCost = 4, kLeastCost = 8;

// W: width class of d (64, 128, 256).
template <typename T, int W> struct Form {
    static constexpr int ROW = W * (int)sizeof(T), ROWS = ROW == 1024 ? 8 : 16;   // bytes of a row in shared memory; rows of a tile
    static constexpr int TILE = 2 * ROWS * ROW, RING = kStages * TILE;             // K's rows, then V's
    static constexpr int WEIGHTS = sizeof(T) == 4 ? 640 : 0;                       // fp32: a tile's weights
    static constexpr int SHARED = kAttnWarps * (RING + WEIGHTS);
    static constexpr int CTAS = SHARED <= 56 * 1024 ? 4 : SHARED <= 113 * 1024 ? 2 : 1;   // of an SM
};

struct Side {   // K or V: byte strides
    const char *data;
    unsigned ld, sh, sp;
};
template <typename T> struct AttnArgs {
    Tables t;
    Tokens tok;
    const T *q;
    long long q_ld, q_sh;
    int M, heads, kv_heads, d, page, pages, group, blocks, pack;   // blocks: of a key head's queries; pack: most tokens of a unit, a power of two
    Side k, v;
    const int *lists;        // [M][kv_heads][keep] or NULL
    int keep;
    float scale;
    Div by_page, by_heads;   // by_heads: heads of one token in a unit
    bool q_pairs, q_fours, out_pairs, by_unit;        // by_unit: `joins` are indexed by unit, else by warp
    T *out;
    long long out_ld, out_sh;
    float *lse;
    float *part;             // two of [queries of a unit][W] per warp: of the unit it begins in the middle of, of the one it leaves in the middle
    float2 *part_ml;         // (maximum to base 2, sum) of each
    int4 *joins;             // (unit, first warp, last warp, queries) of units in several shares; first warp -1: none
};

// The tokens of a unit: `n` from token i on (0: token i belongs to the unit of one before it).  They are of one request, and do not cross multiples of
// `pack`.  most, least: of the positions that they see.
struct Pack { int n, most, least; };
template <typename T> __device__ __forceinline__ Pack pack_of(const AttnArgs<T> &a, int i)
{
    Pack p;
    p.most = p.least = seen_of(a.tok, a.t, a.page, i);
    p.n = 1;
    if (a.pack == 1) return p;
    const int r = a.tok.rows[i], end = min((i & -a.pack) + a.pack, a.M);   // (packs of several tokens: rows are given)
    if ((i & (a.pack - 1)) && a.tok.rows[i - 1] == r) { p.n = 0; return p; }
    while (i + p.n < end && a.tok.rows[i + p.n] == r) {
        const int s = seen_of(a.tok, a.t, a.page, i + p.n);
        p.most = max(p.most, s);
        p.least = min(p.least, s);
        ++p.n;
    }
    return p;
}
template <int ROWS, typename T> __device__ __forceinline__ int tiles_of(const AttnArgs<T> &a, const Pack &p)
{
    const int n = a.lists && p.most ? a.keep * a.page : p.most;
    return max(1, (int)((n + (ROWS - 1ll)) / ROWS));   // (tokens that see nothing have a tile of nothing)
}

// 16 bytes, the first n of them from memory and zeros behind.
__device__ __forceinline__ void copy16(unsigned to, const void *from, int n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
}
__device__ __forceinline__ unsigned long long times(int a, unsigned b) { return (unsigned long long)(unsigned)a * b; }

// The rows of a unit's tiles.  ALIGNED: pages are whole tiles, so a tile lies in one page and its rows are a stride apart; else lane r finds row r.
template <typename T, int W, bool ALIGNED> struct Rows {
    using F = Form<T, W>;
    static constexpr int N = 16 / sizeof(T), CHUNKS = F::ROW / 16, PER = F::ROWS * CHUNKS / 32;   // elements of 16 bytes; of a row; copies of a lane
    static constexpr int AT_ONCE = CHUNKS > 32 ? 1 : 32 / CHUNKS;                                   // rows of a warp's copy (1024 bytes: half of one)
    const AttnArgs<T> &a;
    const int *table, *list;
    const char *k, *v;
    int seen, n, lane, size0, size1;   // n: positions of the unit's line; bytes that this lane's copies take (rows of 1024 bytes: two kinds)
    unsigned place;

    __device__ __forceinline__ Rows(const AttnArgs<T> &a_, int i, int g, int seen_, int lane_) : a(a_), seen(seen_), lane(lane_)
    {
        table = a.t.entries + (seen ? row_of(a.tok, i) * a.t.ld : 0);
        list = a.lists ? a.lists + ((long long)i * a.kv_heads + g) * a.keep : nullptr;
        n = seen == 0 ? 0 : list ? a.keep * a.page : seen;
        const int row = lane / CHUNKS, chunk = lane % CHUNKS;
        size0 = min(max((a.d - chunk * N) * (int)sizeof(T), 0), 16);
        size1 = CHUNKS > 32 ? min(max((a.d - (lane + 32) * N) * (int)sizeof(T), 0), 16) : size0;
        k = a.k.data + times(g, a.k.sh);
        v = a.v.data + times(g, a.v.sh);
        if (ALIGNED) {   // (what a lane does not read is not pointed to either)
            k += times(row, a.k.ld);
            v += times(row, a.v.ld);
        }
        k += size0 ? chunk * 16 : 0;
        v += size0 ? chunk * 16 : 0;
        // bfloat16: a row's 16-byte pieces are turned by the row, so that eight rows' pieces at one place lie in different banks
        place = row * F::ROW + (sizeof(T) == 2 ? chunk ^ row : chunk) * 16;
    }
    // In three steps, a tile apart, so that nothing waits for them: the page's index in the table, the page, the copies.
    struct At { int c, r, held; };   // index in the table (-1: nothing is there), row of the page (ALIGNED: the tile's first), page
    __device__ __forceinline__ At index(int tile) const
    {
        At x;
        const unsigned p = (unsigned)tile * F::ROWS + (ALIGNED ? 0 : lane % F::ROWS);
        x.c = -1; x.r = 0; x.held = -1;
        if (p < (unsigned)n) {
            x.c = (int)a.by_page(p);
            x.r = (int)p - x.c * a.page;
            if (list) x.c = list[x.c];
        }
        return x;
    }
    __device__ __forceinline__ void page(At &x) const
    {
        if (list && (x.c < 0 || x.c * (long long)a.page + x.r >= seen)) x.c = -1;
        x.held = x.c < 0 ? -1 : table[x.c];
    }
    static __device__ __forceinline__ unsigned to_of(unsigned to, unsigned place, int i)   // of copy i
    {
        if (CHUNKS > 32) return to + (i / 2) * F::ROW + (i & 1) * 512 + place;
        return to + i * AT_ONCE * F::ROW + (sizeof(T) == 2 ? place ^ ((i * AT_ONCE & 7) * 16) : place);
    }
    // Begins the copies of a tile; which of its rows are there.
    __device__ __forceinline__ unsigned copy(const At &x, unsigned to) const
    {
        constexpr unsigned ALL = (1u << F::ROWS) - 1;
        const bool on = (unsigned)x.held < (unsigned)a.pages;
        if (ALIGNED) {
            if (!on) return 0;
            const int rows = seen - (x.c * a.page + x.r);   // (c * page + r < seen)
            const char *kr = k + times(x.held, a.k.sp) + times(x.r, a.k.ld), *vr = v + times(x.held, a.v.sp) + times(x.r, a.v.ld);
            const unsigned long long k_step = (unsigned long long)a.k.ld * AT_ONCE, v_step = (unsigned long long)a.v.ld * AT_ONCE;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int row = CHUNKS > 32 ? i / 2 : i * AT_ONCE + lane / CHUNKS, half = CHUNKS > 32 ? i & 1 : 0;
                const int whole = half ? size1 : size0, size = row < rows ? whole : 0, more = half && size1 ? 512 : 0;
                copy16(to_of(to, place, i), kr + more, size);
                copy16(to_of(to, place, i) + F::ROWS * F::ROW, vr + more, size);
                if (CHUNKS <= 32 || half) { kr += k_step; vr += v_step; }
            }
            return rows >= F::ROWS ? ALL : (1u << rows) - 1;
        } else {
            const unsigned there = __ballot_sync(~0u, on) & ALL;
            if (!there) return 0;
            // lanes below 16 find K's rows, the others V's
            const unsigned long long mine = !on ? 0 : lane < 16 ? times(x.held, a.k.sp) + times(x.r, a.k.ld) : times(x.held, a.v.sp) + times(x.r, a.v.ld);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int row = CHUNKS > 32 ? i / 2 : i * AT_ONCE + lane / CHUNKS, half = CHUNKS > 32 ? i & 1 : 0;
                const int size = there >> row & 1 ? (half ? size1 : size0) : 0, more = half && size1 ? 512 : 0;
                copy16(to_of(to, place, i), k + __shfl_sync(~0u, mine, row) + more, size);
                copy16(to_of(to, place, i) + F::ROWS * F::ROW, v + __shfl_sync(~0u, mine, row + 16) + more, size);
            }
            return there;
        }
    }
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void load_matrices(unsigned (&x)[4], unsigned at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_transposed(unsigned (&x)[4], unsigned at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ unsigned transposed(unsigned x)   // of 8 x 8 16-bit numbers, two in a lane
{
    unsigned y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Where a unit's queries are: query c is head first + c % heads of token i + c / heads.
template <typename T> struct Queries {
    const AttnArgs<T> &a;
    int i, first, n;
    __device__ __forceinline__ void of(int c, int &token, int &head) const
    {
        const int j = (int)a.by_heads((unsigned)c);
        token = i + j;
        head = first + c - j * (int)a.by_heads.d;
    }
    __device__ __forceinline__ const T *query(int c) const { int t, h; of(c, t, h); return a.q + t * a.q_ld + h * a.q_sh; }
    __device__ __forceinline__ T *out(int c) const { int t, h; of(c, t, h); return a.out + t * a.out_ld + h * a.out_sh; }
    __device__ __forceinline__ float *lse(int c) const { int t, h; of(c, t, h); return a.lse + (long long)t * a.heads + h; }
    __device__ __forceinline__ int sees(int c) const
    {
        if (c >= n) return INT_MAX;
        int t, h;
        of(c, t, h);
        return seen_of(a.tok, a.t, a.page, t);
    }
};
__device__ __forceinline__ float lse_of(float base, float sum) { return sum == 0.f ? -CUDART_INF_F : (base + log2f(sum)) * attn::kLn2; }
constexpr float kAhead = 8.f;   // the reference of the exponentials follows the maximum when that is 2^8 ahead of it

// What a warp holds of a unit, bfloat16: the tile's rows are the long side of the products (S^T = K Q^T, O^T = V^T P^T), the queries the side of eight, so
// that no more than the queries there are is padded, and K and V come straight from their rows by ldmatrix.
// A weight goes into its product as two bfloat16 that make up 16 bits of it; what bounds the kernel leaves the tensor cores time for that.  With an infinity in V
// the lower part would make 0 * inf or inf - inf of it, so a unit whose sums are not finite is taken again with the upper part alone.
template <int W, int NT> struct Tile16 {
    static constexpr int QUERIES = 8 * NT, KS = W / 16;
    unsigned q[KS][NT][2];
    float o[KS][NT][4];       // [columns 16 x ..][queries 8 x ..]: columns g, g + 8 (pairs), queries 2 t, 2 t + 1
    float base[NT][2], ahead[NT][2], sum[NT][2];   // of queries 2 t, 2 t + 1; ahead: by how much a logit may exceed base (-inf: none has been met)
    int sees[NT][2];
    bool lower;

    __device__ __forceinline__ void begin(const Queries<Bf16> &u, int lane, bool alike)
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int m = 0; m < NT; ++m) {
            const int c = m * 8 + g;
            const Bf16 *p = c < u.n ? u.query(c) : nullptr;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int e = s * 16 + x * 8 + t * 2;
                    unsigned y = 0;
                    if (p) {
                        if (u.a.q_pairs && e + 1 < u.a.d) y = *reinterpret_cast<const unsigned *>(p + e);
                        else y = (e < u.a.d ? p[e].bits : 0) | (unsigned)(e + 1 < u.a.d ? p[e + 1].bits : 0) << 16;
                    }
                    q[s][m][x] = y;
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) sees[m][e] = alike ? INT_MAX : u.sees(m * 8 + 2 * t + e);
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int m = 0; m < NT; ++m) {
#pragma unroll
            for (int e = 0; e < 2; ++e) { ahead[m][e] = -CUDART_INF_F; base[m][e] = 0.f; sum[m][e] = 0.f; }
#pragma unroll
            for (int s = 0; s < KS; ++s) o[s][m][0] = o[s][m][1] = o[s][m][2] = o[s][m][3] = 0.f;
        }
    }
    // there: the tile's rows that are there; first: the position of its row 0, or -1 if all queries see all of them.
    __device__ __forceinline__ void take(unsigned at, unsigned there, int first, float scale2, int lane, float *)
    {
        using F = Form<Bf16, W>;
        float x[NT][4] = {}, y[NT][4] = {};   // two sums, so that half as many products wait for one another
        {
            const int row = lane & 15;
            const unsigned from = at + row * F::ROW, turn = ((lane >> 4) ^ (row & 7)) * 16;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                unsigned k[4];
                load_matrices(k, from + (turn ^ (s & 3) * 32) + (s >> 2) * 128);
#pragma unroll
                for (int m = 0; m < NT; ++m) mma_bf16(s & 1 ? y[m] : x[m], k, q[s][m][0], q[s][m][1]);
            }
        }
        const int g = lane >> 2;
        bool move = false;
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[m][e] += y[m][e];
                x[m][e] = fmaf(x[m][e], scale2, -base[m][e & 1]);
            }
        if (there != 0xffffu || first >= 0) {
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = e < 2 ? g : g + 8;
                    if (!(there >> row & 1) || (first >= 0 && first + row >= sees[m][e & 1])) x[m][e] = -CUDART_INF_F;
                }
        }
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e) move |= fmaxf(x[m][e], x[m][e + 2]) > ahead[m][e];
        if (__any_sync(~0u, move)) {
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float by = fmaxf(x[m][e], x[m][e + 2]);
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) by = fmaxf(by, __shfl_xor_sync(~0u, by, w));
                    float fall = 1.f;
                    if (by == -CUDART_INF_F) by = 0.f;
                    else if (ahead[m][e] == kAhead) fall = attn::ex2(-(by = fmaxf(by, 0.f)));
                    else ahead[m][e] = kAhead;   // the first logit, which may lie far below 0
                    base[m][e] += by;
                    x[m][e] -= by;
                    x[m][e + 2] -= by;
                    sum[m][e] *= fall;
#pragma unroll
                    for (int s = 0; s < KS; ++s) { o[s][m][e] *= fall; o[s][m][e + 2] *= fall; }
                }
        }
        unsigned high[NT][2], low[NT][2];
#pragma unroll
        for (int m = 0; m < NT; ++m) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[m][e] = attn::ex2(x[m][e]);
                sum[m][e & 1] += x[m][e];
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const unsigned u = attn::bf16x2(x[m][2 * j], x[m][2 * j + 1]);
                high[m][j] = transposed(u);
                low[m][j] = transposed(attn::bf16x2(x[m][2 * j] - __uint_as_float(u << 16), x[m][2 * j + 1] - __uint_as_float(u & 0xffff0000u)));
            }
        }
        const int row = (lane >> 4) * 8 + (lane & 7);
        const unsigned from = at + (F::ROWS + row) * F::ROW, turn = ((lane >> 3 & 1) ^ (lane & 7)) * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            unsigned v[4];
            load_transposed(v, from + (turn ^ (s & 3) * 32) + (s >> 2) * 128);
#pragma unroll
            for (int m = 0; m < NT; ++m) {
                mma_bf16(o[s][m], v, high[m][0], high[m][1]);
                if (lower) mma_bf16(o[s][m], v, low[m][0], low[m][1]);
            }
        }
    }
    // True: to be taken again.
    __device__ __forceinline__ bool again()
    {
        bool odd = false;
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= !(fabsf(o[s][m][e]) <= 3.402823466e38f);
        odd = __any_sync(~0u, odd) && lower;
        if (odd) lower = false;
        return odd;
    }
    __device__ __forceinline__ void total()
    {
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) sum[m][e] += __shfl_xor_sync(~0u, sum[m][e], w);
    }
    __device__ __forceinline__ void write(const Queries<Bf16> &u, int lane)
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int m = 0; m < NT; ++m) {
            if (m * 8 >= u.n) break;
            float f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                f[e] = sum[m][e] == 0.f ? 0.f : 1.f / sum[m][e];
                const int c = m * 8 + 2 * t + e;
                if (g == 0 && c < u.n) *u.lse(c) = lse_of(base[m][e], sum[m][e]);
            }
            const int c = m * 8 + g;
            Bf16 *out = c < u.n ? u.out(c) : nullptr;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    // columns by queries to queries by columns: this lane's query g, columns 2 t and 2 t + 1
                    const unsigned y = transposed(attn::bf16x2(o[s][m][2 * j] * f[0], o[s][m][2 * j + 1] * f[1]));
                    const int e = s * 16 + j * 8 + 2 * t;
                    if (!out) continue;
                    if (u.a.out_pairs && e + 1 < u.a.d) { *reinterpret_cast<unsigned *>(out + e) = y; continue; }
                    if (e < u.a.d) out[e].bits = (unsigned short)y;
                    if (e + 1 < u.a.d) out[e + 1].bits = (unsigned short)(y >> 16);
                }
        }
    }
    __device__ __forceinline__ void leave(float *part, float2 *ml, int queries, int lane)
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = m * 8 + 2 * t + e;
                if (c >= queries) continue;
                if (g == 0) ml[c] = make_float2(ahead[m][e] == kAhead ? base[m][e] : -CUDART_INF_F, sum[m][e]);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    part[c * W + s * 16 + g] = o[s][m][e];
                    part[c * W + s * 16 + g + 8] = o[s][m][e + 2];
                }
            }
    }
};

// The same in fp32, on the CUDA cores, two sums an instruction.  A lane of S has a query (lane & 7) and every fourth 16 bytes of it in registers, and
// reads those of each row of K along with the seven other queries' lanes; four lanes' sums then go to one of them for each row.  A lane of O has W / 32 columns
// of all eight queries and reads the weights, which pass through shared memory.
template <int W> struct Tile32 {
    static constexpr int QUERIES = 8, ROWS = Form<float, W>::ROWS, MINE = ROWS / 4, COLS = W / 32;
    uint64_t q[W / 16][2], o[4][COLS];   // o: pairs of queries, columns
    float base, ahead, sum;
    int sees;
    bool lower;

    __device__ __forceinline__ void begin(const Queries<float> &u, int lane, bool alike)
    {
        const int c = lane & 7, part = lane >> 3;
        const float *p = c < u.n ? u.query(c) : nullptr;
        sees = alike ? INT_MAX : u.sees(c);
#pragma unroll
        for (int i = 0; i < W / 16; ++i) {
            const int e = (i * 4 + part) * 4;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (p) {
                if (u.a.q_fours && e + 3 < u.a.d) {
                    x = *reinterpret_cast<const float4 *>(p + e);
                } else {
                    if (e < u.a.d) x.x = p[e];
                    if (e + 1 < u.a.d) x.y = p[e + 1];
                    if (e + 2 < u.a.d) x.z = p[e + 2];
                    if (e + 3 < u.a.d) x.w = p[e + 3];
                }
            }
            q[i][0] = attn::two(x.x, x.y);
            q[i][1] = attn::two(x.z, x.w);
        }
    }
    __device__ __forceinline__ void clear()
    {
        ahead = -CUDART_INF_F; base = 0.f; sum = 0.f;
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int c = 0; c < COLS; ++c) o[h][c] = 0;
    }
    static __device__ __forceinline__ int weights_of(int row) { return row * 8 + row / MINE * 8; }   // (four rows that are written at once: different banks)
    __device__ __forceinline__ void take(unsigned at, unsigned there, int first, float scale2, int lane, float *weights)
    {
        using F = Form<float, W>;
        const int part = lane >> 3;
        float s[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            uint64_t x = 0, y = 0;
#pragma unroll
            for (int i = 0; i < W / 16; ++i) {
                uint64_t k0, k1;
                asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(k0), "=l"(k1) : "r"(at + r * F::ROW + (i * 4 + part) * 16) : "memory");
                x = attn::fma2(q[i][0], k0, x);
                y = attn::fma2(q[i][1], k1, y);
            }
            float u, v, w, z;
            attn::split(x, u, v);
            attn::split(y, w, z);
            s[r] = (u + w) + (v + z);
        }
        // four lanes' sums of every row -> one lane's: rows part * MINE ...
        const bool up = part & 2, odd = part & 1;
#pragma unroll
        for (int r = 0; r < ROWS / 2; ++r) {
            const float give = up ? s[r] : s[r + ROWS / 2], keep = up ? s[r + ROWS / 2] : s[r];
            s[r] = keep + __shfl_xor_sync(~0u, give, 16);
        }
        bool move = false;
#pragma unroll
        for (int r = 0; r < MINE; ++r) {
            const float give = odd ? s[r] : s[r + MINE], keep = odd ? s[r + MINE] : s[r];
            s[r] = fmaf(keep + __shfl_xor_sync(~0u, give, 8), scale2, -base);
            const int row = part * MINE + r;
            if (!(there >> row & 1) || (first >= 0 && first + row >= sees)) s[r] = -CUDART_INF_F;
            move |= s[r] > ahead;
        }
        if (__any_sync(~0u, move)) {
            float by = s[0];
#pragma unroll
            for (int r = 1; r < MINE; ++r) by = fmaxf(by, s[r]);
            by = fmaxf(by, __shfl_xor_sync(~0u, by, 8));
            by = fmaxf(by, __shfl_xor_sync(~0u, by, 16));
            float fall = 1.f;
            if (by == -CUDART_INF_F) by = 0.f;
            else if (ahead == kAhead) fall = attn::ex2(-(by = fmaxf(by, 0.f)));
            else ahead = kAhead;
            base += by;
            sum *= fall;
#pragma unroll
            for (int r = 0; r < MINE; ++r) s[r] -= by;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const uint64_t f = attn::two(__shfl_sync(~0u, fall, 2 * h), __shfl_sync(~0u, fall, 2 * h + 1));
#pragma unroll
                for (int c = 0; c < COLS; ++c) o[h][c] = attn::mul2(o[h][c], f);
            }
        }
#pragma unroll
        for (int r = 0; r < MINE; ++r) {
            s[r] = attn::ex2(s[r]);
            sum += s[r];
            weights[weights_of(part * MINE + r) + (lane & 7)] = s[r];
        }
        __syncwarp();
        const unsigned v_at = at + ROWS * F::ROW;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float v[COLS];
            if constexpr (COLS == 2) {
                asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(v_at + r * F::ROW + lane * 8) : "memory");
            } else {
#pragma unroll
                for (int c = 0; c < COLS; c += 4)
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[c]), "=f"(v[c + 1]), "=f"(v[c + 2]), "=f"(v[c + 3])
                                 : "r"(v_at + r * F::ROW + lane * 16 + c * 128) : "memory");
            }
            const ulonglong2 *p = reinterpret_cast<const ulonglong2 *>(weights + weights_of(r));
            const ulonglong2 p0 = p[0], p1 = p[1];
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const uint64_t x = attn::two(v[c], v[c]);
                o[0][c] = attn::fma2(p0.x, x, o[0][c]);
                o[1][c] = attn::fma2(p0.y, x, o[1][c]);
                o[2][c] = attn::fma2(p1.x, x, o[2][c]);
                o[3][c] = attn::fma2(p1.y, x, o[3][c]);
            }
        }
    }
    __device__ __forceinline__ bool again() { return false; }
    __device__ __forceinline__ void total()
    {
        sum += __shfl_xor_sync(~0u, sum, 8);
        sum += __shfl_xor_sync(~0u, sum, 16);
    }
    static __device__ __forceinline__ int column(int c, int lane) { return COLS == 2 ? lane * 2 + c : lane * 4 + c / 4 * 128 + c % 4; }
    __device__ __forceinline__ void write(const Queries<float> &u, int lane)
    {
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        if (lane < u.n) *u.lse(lane) = lse_of(base, sum);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            if (2 * h >= u.n) break;
            const float f0 = __shfl_sync(~0u, f, 2 * h), f1 = __shfl_sync(~0u, f, 2 * h + 1);
            float *out0 = u.out(2 * h), *out1 = 2 * h + 1 < u.n ? u.out(2 * h + 1) : nullptr;
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const int e = column(c, lane);
                float x, y;
                attn::split(o[h][c], x, y);
                if (e < u.a.d) out0[e] = x * f0;
                if (e < u.a.d && out1) out1[e] = y * f1;
            }
        }
    }
    __device__ __forceinline__ void leave(float *part, float2 *ml, int queries, int lane)
    {
        if (lane < queries) ml[lane] = make_float2(ahead == kAhead ? base : -CUDART_INF_F, sum);
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                float x, y;
                attn::split(o[h][c], x, y);
                if (2 * h < queries) part[2 * h * W + column(c, lane)] = x;
                if (2 * h + 1 < queries) part[(2 * h + 1) * W + column(c, lane)] = y;
            }
    }
};
template <typename T, int W, int NT> struct TileOf { using type = Tile16<W, NT>; };
template <int W, int NT> struct TileOf<float, W, NT> { using type = Tile32<W>; };

template <typename T, int W, int NT, bool ALIGNED>
__global__ void __launch_bounds__(kAttnWarps * 32, Form<T, W>::CTAS) paged_attention_kernel(const AttnArgs<T> a)
{
    using F = Form<T, W>;
    using Tile = typename TileOf<T, W, NT>::type;
    extern __shared__ __align__(128) char shared[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, me = blockIdx.x * kAttnWarps + warp;
    const int units = a.kv_heads * a.blocks;   // of a token
    char *ring = shared + warp * F::RING;
    float *weights = reinterpret_cast<float *>(shared + kAttnWarps * F::RING + warp * F::WEIGHTS);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const auto cost = [&](int i) {
        const Pack p = pack_of(a, i);
        return p.n ? (long long)(tiles_of<F::ROWS>(a, p) + kUnitCost) * units : 0ll;
    };
    Share w;
    if (!deal<kAttnWarps * 32>(a.M, cost, gridDim.x * kAttnWarps, me, kLeastCost, w)) {
        if (!a.by_unit && lane == 0) a.joins[me] = make_int4(0, -1, 0, 0);
        return;
    }
    int4 join = make_int4(0, -1, 0, 0);
    const float scale2 = a.scale * attn::kLog2e;
    Pack p = pack_of(a, w.row);
    int i = w.row, tiles = tiles_of<F::ROWS>(a, p), unit;   // unit of the token; what of it lies before this warp's share
    long long before;
    if (w.rest >> 31) {
        unit = (int)(w.rest / (tiles + kUnitCost));
        before = w.rest - (long long)unit * (tiles + kUnitCost);
    } else {
        unit = (int)w.rest / (tiles + kUnitCost);
        before = (int)w.rest - unit * (tiles + kUnitCost);
    }
    Tile x;
    for (long long at = w.lo;;) {
        // position `at` of the line is `before` behind the unit's begin; tile t of the unit lies at kUnitCost + t
        const long long begin = at - before, end = min(begin + tiles + kUnitCost, w.hi);
        const int first = (int)max(before - kUnitCost, 0ll), last = (int)(end - begin) - kUnitCost;   // tiles
        if (last > first) {
            const int g = unit / a.blocks, b = unit - g * a.blocks;
            const Queries<T> u{a, i, g * a.group + b * Tile::QUERIES, a.pack > 1 ? p.n * a.group : min(Tile::QUERIES, a.group - b * Tile::QUERIES)};
            const Rows<T, W, ALIGNED> rows(a, i, g, p.most, lane);
            // a tile's index is found four tiles ahead of its use, its page three, and its copies begin two ahead
            typename Rows<T, W, ALIGNED>::At now = rows.index(first), next = rows.index(first + 1), third = rows.index(first + 2), fourth = rows.index(first + 3);
            x.begin(u, lane, p.n == 1);
            x.lower = true;
            do {
                x.clear();
                unsigned there, there1, there2;
                const unsigned to = (unsigned)__cvta_generic_to_shared(ring);
                rows.page(now);
                rows.page(next);
                rows.page(third);
                there = rows.copy(now, to);
                asm volatile("cp.async.commit_group;" ::: "memory");
                there1 = first + 1 < last ? rows.copy(next, to + F::TILE) : 0;
                asm volatile("cp.async.commit_group;" ::: "memory");
                int stage = 0;
                for (int j = first; j < last; ++j) {
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    __syncwarp();
                    const int free = stage == 0 ? 2 : stage - 1;
                    there2 = j + 2 < last ? rows.copy(third, to + free * F::TILE) : 0;
                    asm volatile("cp.async.commit_group;" ::: "memory");
                    third = fourth;
                    rows.page(third);
                    fourth = rows.index(j + 4);
                    if (there) x.take(to + stage * F::TILE, there, (j + 1) * F::ROWS > p.least && p.n > 1 ? j * F::ROWS : -1, scale2, lane, weights);
                    there = there1;
                    there1 = there2;
                    stage = stage == 2 ? 0 : stage + 1;
                    __syncwarp();
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                __syncwarp();
                if (!x.again()) break;
                now = rows.index(first); next = rows.index(first + 1); third = rows.index(first + 2); fourth = rows.index(first + 3);
            } while (true);
            x.total();
            const int id = i * units + unit;
            const bool all = first == 0 && last == tiles;
            if (all) {
                x.write(u, lane);
            } else {
                const long long slot = me * 2ll + (first == 0);
                x.leave(a.part + slot * Tile::QUERIES * W, a.part_ml + slot * Tile::QUERIES, u.n, lane);
                if (first == 0) join = make_int4(id, me, (int)((begin + tiles + kUnitCost - 1) / w.share), u.n);   // (the warp that the last tile lies with)
            }
            if (first == 0 && a.by_unit && lane < p.n) a.joins[id + lane * units] = lane == 0 && !all ? join : make_int4(0, -1, 0, 0);
        }
        at = end;
        if (at >= w.hi) break;
        before = 0;
        if (++unit == units) {
            unit = 0;
            if ((i += p.n) >= a.M) break;   // (not with lengths that stay as they are)
            p = pack_of(a, i);
            tiles = tiles_of<F::ROWS>(a, p);
        }
    }
    if (!a.by_unit && lane == 0) a.joins[me] = join;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Joins the parts of units in several shares.  WARPS: warps that take a query of an entry of `joins`, kJoinAt parts of it at a time each, whose results are
// joined in order; with one the CTA takes eight queries.
constexpr int kJoinAt = 10;
template <typename T, int W, int WARPS>
__global__ void __launch_bounds__(WARPS == 1 ? 256 : WARPS * 32) paged_join_kernel(const AttnArgs<T> a, int queries)   // queries: of a unit, at most
{
    constexpr int V = W == 256 ? 2 : 1, AT = W == 256 ? kJoinAt / 2 : kJoinAt;   // V: groups of four columns of a lane
    __shared__ float sums[WARPS][W], weight[WARPS], highs[WARPS];
    const int warp = WARPS == 1 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int4 j = a.joins[blockIdx.x];
    const int m = WARPS == 1 ? blockIdx.y * 8 + (threadIdx.x >> 5) : blockIdx.y;
    if (j.y < 0 || m >= j.w) return;
    const int units = a.kv_heads * a.blocks, i = j.x / units, unit = j.x - i * units, g = unit / a.blocks, b = unit - g * a.blocks;
    const Queries<T> u{a, i, g * a.group + b * queries, j.w};
    float x[V][4] = {}, high = -CUDART_INF_F, l = 0.f;
    for (int p = j.y + warp; p <= j.z; p += WARPS * AT) {
        float y[AT][V][4];
        float2 ml[AT];
#pragma unroll
        for (int k = 0; k < AT; ++k) {
            const int c = p + k * WARPS;
            ml[k] = make_float2(-CUDART_INF_F, 0.f);
            if (c <= j.z) {
                const long long slot = (c * 2ll + (c == j.y)) * queries + m;
                ml[k] = a.part_ml[slot];
#pragma unroll
                for (int v = 0; v < V; ++v) attn::load_part(a.part + slot * W, (lane + 32 * v) * 4, W, y[k][v]);
            }
        }
        float to = high;
#pragma unroll
        for (int k = 0; k < AT; ++k) to = fmaxf(to, ml[k].x);
        const float ref = to == -CUDART_INF_F ? 0.f : to, fall = attn::ex2(high - ref);
        high = to;
        l *= fall;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int k = 0; k < 4; ++k) x[v][k] *= fall;
#pragma unroll
        for (int k = 0; k < AT; ++k) {
            if (p + k * WARPS > j.z) break;
            const float f = attn::ex2(ml[k].x - ref);
            l = fmaf(ml[k].y, f, l);
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[v][e] = fmaf(f, y[k][v][e], x[v][e]);
        }
    }
    if constexpr (WARPS == 1) {
        const float f = l == 0.f ? 0.f : 1.f / l;
        T *out = u.out(m);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if ((lane + 32 * v) * 4 + e < a.d) attn::narrow(x[v][e] * f, out[(lane + 32 * v) * 4 + e]);
        if (lane == 0) *u.lse(m) = lse_of(high, l);
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if ((lane + 32 * v) * 4 < W) *reinterpret_cast<float4 *>(&sums[warp][(lane + 32 * v) * 4]) = make_float4(x[v][0], x[v][1], x[v][2], x[v][3]);
        if (lane == 0) { weight[warp] = l; highs[warp] = high; }
        __syncthreads();
        if (threadIdx.x >= W) return;
        high = -CUDART_INF_F;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) high = fmaxf(high, highs[w]);
        const float ref = high == -CUDART_INF_F ? 0.f : high;
        float y = 0.f;
        l = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = attn::ex2(highs[w] - ref);
            l = fmaf(f, weight[w], l);
            y = fmaf(f, sums[w][threadIdx.x], y);
        }
        if (threadIdx.x < a.d) attn::narrow(l == 0.f ? 0.f : y / l, u.out(m)[threadIdx.x]);
        if (threadIdx.x == 0) *u.lse(m) = lse_of(high, l);
    }
}

}  // namespace paged
}  // namespace b2sp
