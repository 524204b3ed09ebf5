// Attention of new tokens over a cache in pages.
//
//   s_j = scale q . k_j;  O = sum_j exp(s_j - m) v_j / l,  l = sum_j exp(s_j - m),  lse = m + log l
//
// over the positions j that a token sees, or those of them in the pages that its list names.  Every row of the cache is read once for the heads that
// share it and used 2 to 16 times, so HBM bounds the work and everything else has to keep out of its way.
//
// A unit is a token, a key head and up to 8 (16) of its query heads; its rows come in tiles of kTileRows.  All units' tiles in a line are dealt to the warps
// in equal shares: a warp takes its share by itself, with a ring of tiles of its own in shared memory that asynchronous copies fill two tiles ahead, and
// waits for no other warp.  It knows its share from prefix sums over the tokens, so lengths stay on the device and a long row is spread over the GPU as
// well as many short ones.  Units that end up in several shares leave their sums in the workspace, and a second kernel joins them in order.
// Rows that are not there (behind what is seen, of missing pages) are filled with zeros by the copies instead of read: what memory holds there does not
// enter.
#pragma once
#include "paged.cuh"

namespace b2sp {
namespace paged {

constexpr int kAttnWarps = 4, kStages = 3, kLeastTiles = 4;   // warps of a CTA; tiles of a warp in shared memory; of a share

// W: width class of d (64, 128, 256).
template <typename T, int W> struct Form {
    static constexpr int ROW = W * (int)sizeof(T), ROWS = ROW == 1024 ? 8 : 16;   // bytes of a row in shared memory; rows of a tile
    static constexpr int TILE = 2 * ROWS * ROW, RING = kStages * TILE;             // K's rows, then V's
    static constexpr int WEIGHTS = sizeof(T) == 4 ? 640 : 0;                       // fp32: a tile's weights
    static constexpr int SHARED = kAttnWarps * (RING + WEIGHTS);
    static constexpr int CTAS = SHARED <= 56 * 1024 ? 4 : SHARED <= 113 * 1024 ? 2 : 1;   // of an SM
};

template <typename T> struct AttnArgs {
    Tables t;
    Tokens tok;
    const T *q;
    long long q_ld, q_sh;
    int M, heads, kv_heads, d, page, group, blocks;   // blocks: of a key head's query heads
    Pages<T> k, v;
    const int *lists;        // [M][kv_heads][keep] or NULL
    int keep;
    float scale;
    Div by_page;
    bool q_pairs, q_fours, out_pairs, by_unit;        // by_unit: `joins` are indexed by unit, else by warp
    T *out;
    long long out_ld, out_sh;
    float *lse;
    float *part;             // two of [heads of a unit][W] per warp: of the unit it begins in the middle of, of the one it leaves in the middle
    float2 *part_ml;         // (maximum to base 2, sum) of each
    int4 *joins;             // (unit, first warp, last warp, 0) of units in several shares; first warp -1: none
};

struct Work { int row, unit, tile; };   // token, unit of the token, tile of the unit

template <typename T, int ROWS> __device__ __forceinline__ int tiles_of(const AttnArgs<T> &a, int i, int &seen)
{
    seen = seen_of(a.tok, a.t, a.page, i);
    const int n = a.lists && seen ? a.keep * a.page : seen;
    return max(1, (int)((n + (ROWS - 1ll)) / ROWS));   // (a token that sees nothing has a tile of nothing)
}

// 16 bytes, the first n of them from memory and zeros behind.
__device__ __forceinline__ void copy16(unsigned to, const void *from, int n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
}

// The rows of a unit's tiles.  ALIGNED: pages are whole tiles, so a tile lies in one page and its rows are a stride apart; else lane r finds row r.
template <typename T, int W, bool ALIGNED> struct Rows {
    using F = Form<T, W>;
    static constexpr int N = 16 / sizeof(T), CHUNKS = F::ROW / 16, PER = F::ROWS * CHUNKS / 32;   // elements of 16 bytes; of a row; copies of a lane
    const AttnArgs<T> &a;
    const int *table, *list;
    int seen, n, lane, size0, size1;   // n: positions of the unit's line; bytes that this lane's copies take (rows of 1024 bytes: two kinds)
    long long head_k, head_v;

    __device__ __forceinline__ Rows(const AttnArgs<T> &a_, int i, int g, int seen_, int lane_) : a(a_), seen(seen_), lane(lane_)
    {
        table = a.t.entries + (seen ? row_of(a.tok, i) * a.t.ld : 0);
        list = a.lists ? a.lists + ((long long)i * a.kv_heads + g) * a.keep : nullptr;
        n = seen == 0 ? 0 : list ? a.keep * a.page : seen;
        size0 = min(max((a.d - lane % CHUNKS * N) * (int)sizeof(T), 0), 16);
        size1 = CHUNKS > 32 ? min(max((a.d - (lane + 32) * N) * (int)sizeof(T), 0), 16) : size0;
        head_k = g * a.k.sh;
        head_v = g * a.v.sh;
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
        if (x.c < 0 || x.c * (long long)a.page + x.r >= seen) x.c = -1;
        x.held = x.c < 0 ? -1 : table[x.c];
    }
    // Begins the copies of a tile; which of its rows are there.
    __device__ __forceinline__ unsigned copy(const At &x, unsigned to) const
    {
        const bool on = (unsigned)x.held < (unsigned)a.k.pages;
        if (ALIGNED) {
            if (!on) return 0;
            const int rows = (int)min((long long)F::ROWS, seen - (x.c * (long long)a.page + x.r));
            const char *k = reinterpret_cast<const char *>(a.k.data + (x.held * a.k.sp + head_k + x.r * a.k.ld)) + lane % CHUNKS * 16;
            const char *v = reinterpret_cast<const char *>(a.v.data + (x.held * a.v.sp + head_v + x.r * a.v.ld)) + lane % CHUNKS * 16;
            const long long k_ld = a.k.ld * (long long)sizeof(T), v_ld = a.v.ld * (long long)sizeof(T);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int row = CHUNKS > 32 ? i / 2 : i * (32 / CHUNKS) + lane / CHUNKS, col = CHUNKS > 32 && (i & 1) ? 512 : 0;
                const int size = row < rows ? (col ? size1 : size0) : 0;
                const unsigned at = to + row * F::ROW + place(row, lane % CHUNKS) + col;
                copy16(at, k + (size ? row * k_ld + col : 0), size);
                copy16(at + F::ROWS * F::ROW, v + (size ? row * v_ld + col : 0), size);
            }
            return rows == F::ROWS ? (1u << F::ROWS) - 1 : (1u << rows) - 1;
        } else {
            const unsigned there = __ballot_sync(~0u, on) & ((1u << F::ROWS) - 1);
            if (!there) return 0;
            const int held = max(x.held, 0);
            // lanes below 16 keep K's rows, the others V's
            const char *mine = lane < 16 ? reinterpret_cast<const char *>(a.k.data + (on ? held * a.k.sp + head_k + x.r * a.k.ld : 0))
                                         : reinterpret_cast<const char *>(a.v.data + (on ? held * a.v.sp + head_v + x.r * a.v.ld : 0));
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int row = CHUNKS > 32 ? i / 2 : i * (32 / CHUNKS) + lane / CHUNKS, col = CHUNKS > 32 && (i & 1) ? 512 : 0;
                const int size = there >> row & 1 ? (col ? size1 : size0) : 0, from = size ? lane % CHUNKS * 16 + col : 0;
                const unsigned at = to + row * F::ROW + place(row, lane % CHUNKS) + col;
                copy16(at, reinterpret_cast<const char *>(__shfl_sync(~0u, (unsigned long long)mine, row)) + from, size);
                copy16(at + F::ROWS * F::ROW, reinterpret_cast<const char *>(__shfl_sync(~0u, (unsigned long long)mine, row + 16)) + from, size);
            }
            return there;
        }
    }
    // Where 16 bytes of a row lie in it.  bfloat16: turned by the row, so that eight rows' bytes at one place lie in different banks.
    static __device__ __forceinline__ int place(int row, int chunk) { return (sizeof(T) == 2 ? chunk ^ (row & 7) : chunk) * 16; }
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

// What a warp holds of a unit, bfloat16: the tile's rows are the long side of the products (S^T = K Q^T, O^T = V^T P^T), the heads the side of eight, so
// that no more than the heads there are is padded, and K and V come straight from their rows by ldmatrix.
// A weight goes into its product as two bfloat16 that make up 16 bits of it; what bounds the kernel leaves the tensor cores time for that.  With an infinity in V
// the lower part would make 0 * inf or inf - inf of it, so a unit whose sums are not finite is taken again with the upper part alone.
template <int W, int NT> struct Tile16 {
    static constexpr int HEADS = 8 * NT, KS = W / 16;
    unsigned q[KS][NT][2];
    float o[KS][NT][4];       // [columns 16 x ..][heads 8 x ..]: columns g, g + 8 (pairs), heads 2 t, 2 t + 1
    float top[NT][2], base[NT][2], sum[NT][2];   // of heads 2 t, 2 t + 1; base: top, or 0 as long as that is -inf
    bool lower;

    __device__ __forceinline__ void begin(const AttnArgs<Bf16> &a, const Bf16 *rows, int heads, int lane)   // queries
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int h = m * 8 + g, e = s * 16 + x * 8 + t * 2;
                    unsigned u = 0;
                    if (h < heads) {
                        const Bf16 *p = rows + h * a.q_sh + e;
                        if (a.q_pairs && e + 1 < a.d) u = *reinterpret_cast<const unsigned *>(p);
                        else u = (e < a.d ? p[0].bits : 0) | (unsigned)(e + 1 < a.d ? p[1].bits : 0) << 16;
                    }
                    q[s][m][x] = u;
                }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int m = 0; m < NT; ++m) {
#pragma unroll
            for (int e = 0; e < 2; ++e) { top[m][e] = -CUDART_INF_F; base[m][e] = 0.f; sum[m][e] = 0.f; }
#pragma unroll
            for (int s = 0; s < KS; ++s) o[s][m][0] = o[s][m][1] = o[s][m][2] = o[s][m][3] = 0.f;
        }
    }
    __device__ __forceinline__ void take(unsigned at, unsigned there, float scale2, int lane, float *)
    {
        using R = Rows<Bf16, W, true>;
        using F = Form<Bf16, W>;
        float x[NT][4] = {}, y[NT][4] = {};   // two sums, so that half as many products wait for one another
        {
            const int row = lane & 15;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                unsigned k[4];
                load_matrices(k, at + row * F::ROW + R::place(row, 2 * s + (lane >> 4)));
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
                x[m][e] = (x[m][e] + y[m][e]) * scale2;
                if (!(there >> (e < 2 ? g : g + 8) & 1)) x[m][e] = -CUDART_INF_F;
                move |= x[m][e] > top[m][e & 1] + 8.f;
            }
        if (__any_sync(~0u, move)) {   // the reference of the exponentials follows the maximum when that is 2^8 ahead
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float to = fmaxf(x[m][e], x[m][e + 2]);
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) to = fmaxf(to, __shfl_xor_sync(~0u, to, w));
                    to = fmaxf(to, top[m][e]);
                    base[m][e] = to == -CUDART_INF_F ? 0.f : to;
                    const float fall = attn::ex2(top[m][e] - base[m][e]);
                    top[m][e] = to;
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
                x[m][e] = attn::ex2(x[m][e] - base[m][e & 1]);
                sum[m][e & 1] += x[m][e];
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const unsigned u = attn::bf16x2(x[m][2 * j], x[m][2 * j + 1]);
                high[m][j] = transposed(u);
                low[m][j] = transposed(attn::bf16x2(x[m][2 * j] - __uint_as_float(u << 16), x[m][2 * j + 1] - __uint_as_float(u & 0xffff0000u)));
            }
        }
        const unsigned v_at = at + F::ROWS * F::ROW;
        const int row = (lane >> 4) * 8 + (lane & 7);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            unsigned v[4];
            load_transposed(v, v_at + row * F::ROW + R::place(row, 2 * s + (lane >> 3 & 1)));
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
    __device__ __forceinline__ void write(const AttnArgs<Bf16> &a, Bf16 *out, float *lse, int heads, int lane)
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int m = 0; m < NT; ++m) {
            float f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                f[e] = sum[m][e] == 0.f ? 0.f : 1.f / sum[m][e];
                const int h = m * 8 + 2 * t + e;
                if (g == 0 && h < heads) lse[h] = sum[m][e] == 0.f ? -CUDART_INF_F : (top[m][e] + log2f(sum[m][e])) * attn::kLn2;
            }
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    // columns by heads to heads by columns: this lane's head g, columns 2 t and 2 t + 1
                    const unsigned u = transposed(attn::bf16x2(o[s][m][2 * j] * f[0], o[s][m][2 * j + 1] * f[1]));
                    const int h = m * 8 + g, c = s * 16 + j * 8 + 2 * t;
                    if (h >= heads) continue;
                    Bf16 *to = out + h * a.out_sh + c;
                    if (a.out_pairs && c + 1 < a.d) { *reinterpret_cast<unsigned *>(to) = u; continue; }
                    if (c < a.d) to[0].bits = (unsigned short)u;
                    if (c + 1 < a.d) to[1].bits = (unsigned short)(u >> 16);
                }
        }
    }
    __device__ __forceinline__ void leave(float *part, float2 *ml, int heads, int lane)
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int h = m * 8 + 2 * t + e;
                if (h >= heads) continue;
                if (g == 0) ml[h] = make_float2(top[m][e], sum[m][e]);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    part[h * W + s * 16 + g] = o[s][m][e];
                    part[h * W + s * 16 + g + 8] = o[s][m][e + 2];
                }
            }
    }
};

// The same in fp32, on the CUDA cores, two sums an instruction.  A lane of S has a head (lane & 7) and every fourth 16 bytes of its query in registers, and
// reads those of each row of K along with the seven other heads' lanes; four lanes' sums then go to one of them for each row.  A lane of O has W / 32 columns of
// all eight heads and reads the weights, which pass through shared memory.
template <int W> struct Tile32 {
    static constexpr int HEADS = 8, ROWS = Form<float, W>::ROWS, MINE = ROWS / 4, COLS = W / 32;
    uint64_t q[W / 16][2], o[4][COLS];   // o: pairs of heads, columns
    float top, base, sum;
    bool lower;

    __device__ __forceinline__ void begin(const AttnArgs<float> &a, const float *rows, int heads, int lane)
    {
        const int h = lane & 7, part = lane >> 3;
#pragma unroll
        for (int i = 0; i < W / 16; ++i) {
            const int e = (i * 4 + part) * 4;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (h < heads) {
                const float *p = rows + h * a.q_sh + e;
                if (a.q_fours && e + 3 < a.d) {
                    x = *reinterpret_cast<const float4 *>(p);
                } else {
                    if (e < a.d) x.x = p[0];
                    if (e + 1 < a.d) x.y = p[1];
                    if (e + 2 < a.d) x.z = p[2];
                    if (e + 3 < a.d) x.w = p[3];
                }
            }
            q[i][0] = attn::two(x.x, x.y);
            q[i][1] = attn::two(x.z, x.w);
        }
    }
    __device__ __forceinline__ void clear()
    {
        top = -CUDART_INF_F; base = 0.f; sum = 0.f;
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int c = 0; c < COLS; ++c) o[h][c] = 0;
    }
    static __device__ __forceinline__ int weights_of(int row) { return row * 8 + row / MINE * 8; }   // (four rows that are written at once: different banks)
    __device__ __forceinline__ void take(unsigned at, unsigned there, float scale2, int lane, float *weights)
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
            s[r] = (keep + __shfl_xor_sync(~0u, give, 8)) * scale2;
            if (!(there >> (part * MINE + r) & 1)) s[r] = -CUDART_INF_F;
            move |= s[r] > top + 8.f;
        }
        if (__any_sync(~0u, move)) {
            float to = top;
#pragma unroll
            for (int r = 0; r < MINE; ++r) to = fmaxf(to, s[r]);
            to = fmaxf(to, __shfl_xor_sync(~0u, to, 8));
            to = fmaxf(to, __shfl_xor_sync(~0u, to, 16));
            base = to == -CUDART_INF_F ? 0.f : to;
            const float fall = attn::ex2(top - base);
            top = to;
            sum *= fall;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const uint64_t f = attn::two(__shfl_sync(~0u, fall, 2 * h), __shfl_sync(~0u, fall, 2 * h + 1));
#pragma unroll
                for (int c = 0; c < COLS; ++c) o[h][c] = attn::mul2(o[h][c], f);
            }
        }
#pragma unroll
        for (int r = 0; r < MINE; ++r) {
            s[r] = attn::ex2(s[r] - base);
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
    __device__ __forceinline__ void write(const AttnArgs<float> &a, float *out, float *lse, int heads, int lane)
    {
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        if (lane < heads) lse[lane] = sum == 0.f ? -CUDART_INF_F : (top + log2f(sum)) * attn::kLn2;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const float f0 = __shfl_sync(~0u, f, 2 * h), f1 = __shfl_sync(~0u, f, 2 * h + 1);
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const int e = column(c, lane);
                float x, y;
                attn::split(o[h][c], x, y);
                if (e < a.d && 2 * h < heads) out[2 * h * a.out_sh + e] = x * f0;
                if (e < a.d && 2 * h + 1 < heads) out[(2 * h + 1) * a.out_sh + e] = y * f1;
            }
        }
    }
    __device__ __forceinline__ void leave(float *part, float2 *ml, int heads, int lane)
    {
        if (lane < heads) ml[lane] = make_float2(top, sum);
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                float x, y;
                attn::split(o[h][c], x, y);
                if (2 * h < heads) part[2 * h * W + column(c, lane)] = x;
                if (2 * h + 1 < heads) part[(2 * h + 1) * W + column(c, lane)] = y;
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
    constexpr int THREADS = kAttnWarps * 32;
    extern __shared__ __align__(128) char shared[];
    __shared__ long long before[THREADS], warps[kAttnWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, me = blockIdx.x * kAttnWarps + warp;
    const int units = a.kv_heads * a.blocks;   // of a token
    const int each = (a.M + THREADS - 1) / THREADS;
    char *ring = shared + warp * F::RING;
    float *weights = reinterpret_cast<float *>(shared + kAttnWarps * F::RING + warp * F::WEIGHTS);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    long long lo, hi, share;
    {
        const int i0 = (int)min((long long)a.M, threadIdx.x * (long long)each), i1 = min(a.M, i0 + each);
        long long n = 0, all;
        int seen;
        for (int i = i0; i < i1; ++i) n += tiles_of<T, F::ROWS>(a, i, seen);
        before[threadIdx.x] = block_before(n, warps, all) * units;
        all *= units;
        share = max((all + gridDim.x * kAttnWarps - 1) / (gridDim.x * kAttnWarps), (long long)kLeastTiles);
        lo = me * share;
        hi = min(lo + share, all);
        __syncthreads();   // `before`
        if (lo >= hi) {
            if (!a.by_unit && lane == 0) a.joins[me] = make_int4(0, -1, 0, 0);
            return;
        }
    }
    // the token that the share begins in
    Work w;
    int seen, tiles;
    {
        int chunk = -1;
#pragma unroll
        for (int j = 0; j < kAttnWarps; ++j) chunk += __popc(__ballot_sync(~0u, before[j * 32 + lane] <= lo));
        long long rest = lo - before[chunk];
        int i = chunk * each;
        for (;;) {   // 32 tokens at a time
            long long n = i + lane < a.M ? (long long)tiles_of<T, F::ROWS>(a, i + lane, seen) * units : 0;
            long long up = n;
#pragma unroll
            for (int x = 1; x < 32; x <<= 1) {
                const long long y = __shfl_up_sync(~0u, up, x);
                if (lane >= x) up += y;
            }
            const unsigned behind = __ballot_sync(~0u, up > rest);
            if (behind) {
                const int k = __ffs(behind) - 1;
                rest -= __shfl_sync(~0u, up - n, k);
                i += k;
                break;
            }
            rest -= __shfl_sync(~0u, up, 31);
            i += 32;
        }
        tiles = tiles_of<T, F::ROWS>(a, i, seen);
        w.row = i;
        w.unit = (int)(rest / tiles);
        w.tile = (int)(rest - (long long)w.unit * tiles);
    }
    int4 join = make_int4(0, -1, 0, 0);
    const float scale2 = a.scale * attn::kLog2e;
    Tile x;
    for (long long left = hi - lo; left > 0;) {
        const int g = w.unit / a.blocks, b = w.unit - g * a.blocks, h0 = g * a.group + b * Tile::HEADS, heads = min(Tile::HEADS, a.group - b * Tile::HEADS);
        const int ends = (int)min((long long)tiles, w.tile + left);
        const Rows<T, W, ALIGNED> rows(a, w.row, g, seen, lane);
        x.begin(a, a.q + w.row * a.q_ld + h0 * a.q_sh, heads, lane);
        x.lower = true;
        do {
            x.clear();
            // a tile's index is found four tiles ahead of its use, its page three, and its copies begin two ahead
            typename Rows<T, W, ALIGNED>::At at = rows.index(w.tile), next = rows.index(w.tile + 1), third = rows.index(w.tile + 2), fourth = rows.index(w.tile + 3);
            unsigned there, there1, there2;
            const unsigned to = (unsigned)__cvta_generic_to_shared(ring);
            rows.page(at);
            rows.page(next);
            rows.page(third);
            there = rows.copy(at, to);
            asm volatile("cp.async.commit_group;" ::: "memory");
            there1 = w.tile + 1 < ends ? rows.copy(next, to + F::TILE) : 0;
            asm volatile("cp.async.commit_group;" ::: "memory");
            int stage = 0;
            for (int j = w.tile; j < ends; ++j) {
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                __syncwarp();
                const int free = stage == 0 ? 2 : stage - 1;
                there2 = j + 2 < ends ? rows.copy(third, to + free * F::TILE) : 0;
                asm volatile("cp.async.commit_group;" ::: "memory");
                third = fourth;
                rows.page(third);
                fourth = rows.index(j + 4);
                if (there) x.take(to + stage * F::TILE, there, scale2, lane, weights);
                there = there1;
                there1 = there2;
                stage = stage == 2 ? 0 : stage + 1;
                __syncwarp();
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
        } while (x.again());
        x.total();
        const int unit = w.row * units + w.unit;
        if (w.tile == 0 && ends == tiles) {
            x.write(a, a.out + w.row * a.out_ld + h0 * a.out_sh, a.lse + (long long)w.row * a.heads + h0, heads, lane);
            if (a.by_unit && lane == 0) a.joins[unit] = make_int4(unit, -1, 0, 0);
        } else {
            const long long slot = me * 2ll + (w.tile == 0);
            x.leave(a.part + slot * Tile::HEADS * W, a.part_ml + slot * Tile::HEADS, heads, lane);
            if (w.tile == 0) {   // the warps that the others lie with: the last tile's is the last one
                join = make_int4(unit, me, (int)((hi - left + tiles - 1) / share), 0);
                if (a.by_unit && lane == 0) a.joins[unit] = join;
            }
        }
        left -= ends - w.tile;
        w.tile = 0;
        if (++w.unit == units && left > 0) {
            w.unit = 0;
            tiles = tiles_of<T, F::ROWS>(a, ++w.row, seen);
        }
    }
    if (!a.by_unit && lane == 0) a.joins[me] = join;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A CTA per entry of `joins` and head of a unit: each warp takes every eighth part (the loads of eight at once), then the warps' sums are joined in order.
constexpr int kJoinWarps = 8;
template <typename T, int W>
__global__ void __launch_bounds__(kJoinWarps * 32) paged_join_kernel(const AttnArgs<T> a, int heads_of_unit)
{
    constexpr int V = W == 256 ? 2 : 1;   // groups of four columns of a lane
    __shared__ float sums[kJoinWarps][W], weight[kJoinWarps], highs[kJoinWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int4 j = a.joins[blockIdx.x];
    const int units = a.kv_heads * a.blocks, row = j.x / units, u = j.x - row * units, g = u / a.blocks, b = u - g * a.blocks, m = blockIdx.y;
    if (j.y < 0 || b * heads_of_unit + m >= a.group) return;
    const int h = g * a.group + b * heads_of_unit + m;
    float x[V][4] = {}, high = -CUDART_INF_F, l = 0.f;
    constexpr int AT = 8;
    for (int p = j.y + warp; p <= j.z; p += kJoinWarps * AT) {
        float y[AT][V][4];
        float2 ml[AT];
#pragma unroll
        for (int i = 0; i < AT; ++i) {
            const int c = p + i * kJoinWarps;
            ml[i] = make_float2(-CUDART_INF_F, 0.f);
#pragma unroll
            for (int v = 0; v < V; ++v) y[i][v][0] = y[i][v][1] = y[i][v][2] = y[i][v][3] = 0.f;
            if (c <= j.z) {
                const long long slot = (c * 2ll + (c == j.y)) * heads_of_unit + m;
                ml[i] = a.part_ml[slot];
#pragma unroll
                for (int v = 0; v < V; ++v) attn::load_part(a.part + slot * W, (lane + 32 * v) * 4, W, y[i][v]);
            }
        }
        float to = high;
#pragma unroll
        for (int i = 0; i < AT; ++i) to = fmaxf(to, ml[i].x);
        const float ref = to == -CUDART_INF_F ? 0.f : to, fall = exp2f(high - ref);
        high = to;
        l *= fall;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int k = 0; k < 4; ++k) x[v][k] *= fall;
#pragma unroll
        for (int i = 0; i < AT; ++i) {
            if (p + i * kJoinWarps > j.z) break;
            const float f = exp2f(ml[i].x - ref);
            l = fmaf(ml[i].y, f, l);
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int k = 0; k < 4; ++k) x[v][k] = fmaf(f, y[i][v][k], x[v][k]);
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if ((lane + 32 * v) * 4 < W) *reinterpret_cast<float4 *>(&sums[warp][(lane + 32 * v) * 4]) = make_float4(x[v][0], x[v][1], x[v][2], x[v][3]);
    if (lane == 0) { weight[warp] = l; highs[warp] = high; }
    __syncthreads();
    high = -CUDART_INF_F;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) high = fmaxf(high, highs[w]);
    const float ref = high == -CUDART_INF_F ? 0.f : high;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) l = fmaf(exp2f(highs[w] - ref), weight[w], l);
    const float f = l == 0.f ? 0.f : 1.f / l;
    for (int e = threadIdx.x; e < a.d; e += kJoinWarps * 32) {
        float y = 0.f;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) y = fmaf(exp2f(highs[w] - ref), sums[w][e], y);
        attn::narrow(y * f, a.out[row * a.out_ld + h * a.out_sh + e]);
    }
    if (threadIdx.x == 0) a.lse[(long long)row * a.heads + h] = l == 0.f ? -CUDART_INF_F : (high + log2f(l)) * attn::kLn2;
}

}  // namespace paged
}  // namespace b2sp
