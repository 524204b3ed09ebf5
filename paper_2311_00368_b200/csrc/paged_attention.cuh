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
// 64 tokens over 1 to 16384 positions, 32 heads over 8, width 128, bfloat16: 2.28 GB in 358 us, 97% of the copy bandwidth; one token over 32768:
// 30.5 us, of which 20.5 are its bytes and the rest is launch, prologue and joining.
// Rows that are not there (behind what is seen, of missing pages) are filled with zeros by the copies instead of read: what memory holds there does not
// enter.  Rows that some queries of a unit see and others do not have a weight of 0 for these, which is nothing unless a value is not finite; see Tile16.
#pragma once
#include "paged.cuh"

namespace b2sp {
namespace paged {

constexpr int kAttnWarps = 4, kStages = 3;   // warps of a CTA; tiles of a warp in shared memory
// A unit costs its tiles and, before the first one, a chain of latencies (lengths, table, rows), as long as about four tiles take: without it warps whose
// shares were many short units took twice as long as the others.  Shares are of at least kLeastCost (2048 positions of one token, 8 key heads: 8.6 us;
// with 4, 6, 8: 9.4, 11.3, 12.9).
constexpr int kUnitCost = 4, kLeastCost = 3;

// W: width class of d (64, 128, 256).
template <typename T, int W, int Q = 8> struct Form {
    static constexpr int ROW = W * (int)sizeof(T), ROWS = ROW == 1024 ? 8 : ROW == 128 ? 32 : 16;   // bytes of a row in shared memory; rows of a tile
    static constexpr int TILE = 2 * ROWS * ROW, RING = kStages * TILE;             // K's rows, then V's
    static constexpr int STORED = sizeof(T) == 4 ? 640 : W == 256 && Q == 16 ? Q * ROW : 0;   // what a warp keeps there beside its ring: fp32 a tile's weights
    static constexpr int SHARED = kAttnWarps * (RING + STORED);
    static constexpr int CTAS = SHARED <= 113 * 1024 ? 2 : 1;   // of an SM
};

struct Side {   // K or V: byte strides
    const char *data;
    unsigned ld, sh, sp;
};
template <typename T> struct AttnArgs {
    Tables t;
    Tokens tok;
    const T *q;
    unsigned q_ld, q_sh;
    int M, heads, kv_heads, d, page, pages, group, blocks, pack;   // blocks: of a key head's queries; pack: most tokens of a unit, a power of two
    Side k, v;
    const int *lists;        // [M][kv_heads][keep] or NULL
    int keep;
    float scale;
    Div by_page, by_heads, by_blocks;   // by_heads: heads of one token in a unit
    bool pairs, fours, by_unit;   // pairs: Q and O begin on four bytes and d is even; fours: Q on sixteen, and fp32's d is a multiple of four; by_unit: `joins` are indexed by unit, else by warp
    T *out;
    unsigned out_ld, out_sh;
    float *lse;
    float *part;             // two of [queries of a unit][W] per warp: of the unit it begins in the middle of, of the one it leaves in the middle
    float2 *part_ml;         // (maximum to base 2, sum) of each
    int *status;
    int4 *joins;             // (unit, first warp, last warp, queries) of units in several shares; first warp -1: none
};

// The tokens of a unit: `n` from token i on.  They are of one request, and do not cross multiples of `pack`.  most, least: of the positions that they see.
struct Pack { int n, most, least; };
// 32 tokens from a multiple of 32 on, one in a lane (`pack` is a power of two below 32, so units do not cross windows).
struct Window { int base, row, seen; };
template <typename T> __device__ __forceinline__ Window window_of(const AttnArgs<T> &a, int base, int lane)
{
    Window w;
    const int i = base + lane;
    w.base = base;
    w.row = INT_MIN;   // (no token)
    w.seen = 0;
    if (i < a.M) {
        const int s = a.tok.seen[i];
        w.row = row_of(a.tok, i);
        w.seen = (unsigned)w.row < (unsigned)a.t.requests ? (int)min((long long)max(s, 0), (long long)a.t.width * a.page) : 0;
    }
    return w;
}
template <typename T> __device__ __forceinline__ Pack pack_of(const AttnArgs<T> &a, const Window &w, int i, int lane)
{
    Pack p;
    const int at = i - w.base, row = __shfl_sync(~0u, w.row, at);
    p.n = 1;
    p.most = p.least = __shfl_sync(~0u, w.seen, at);
    if (a.pack > 1) {
        const unsigned same = __ballot_sync(~0u, w.row == row) >> at;
        p.n = min(min(same == ~0u ? 32 : __ffs(~same) - 1, a.pack - (at & (a.pack - 1))), a.M - i);
        const bool in = lane >= at && lane < at + p.n;
        p.most = __reduce_max_sync(~0u, in ? w.seen : 0);
        p.least = __reduce_min_sync(~0u, in ? w.seen : INT_MAX);
    }
    return p;
}
// Positions of the line of a unit whose tokens see `most`: these, or those of as many entries of the list as there are pages in them.
template <typename T> __device__ __forceinline__ int line_of(const AttnArgs<T> &a, int most)
{
    if (!a.lists) return most;
    const int c = (int)a.by_page((unsigned)most);
    return min(a.keep, c + (c * a.page < most)) * a.page;
}
template <int ROWS, typename T> __device__ __forceinline__ int tiles_of(const AttnArgs<T> &a, int most)
{
    return max(1, (int)(((unsigned)line_of(a, most) + (ROWS - 1u)) / ROWS));   // (tokens that see nothing have a tile of nothing)
}
// What each unit of a window's token `lane` costs: nothing if the token belongs to the units of one before it.
template <int ROWS, typename T> __device__ __forceinline__ int cost_of(const AttnArgs<T> &a, const Window &w, int lane)
{
    int most = w.seen;
    bool begins = true;
    if (a.pack > 1) {
        const int ahead = __shfl_up_sync(~0u, w.row, 1);
        begins = (lane & (a.pack - 1)) == 0 || ahead != w.row;
        const unsigned begin = __ballot_sync(~0u, begins);
        const int mine = 31 - __clz(begin & (2u << lane) - 1);   // where this lane's unit begins
        for (int d = 1; d < a.pack; d *= 2) {
            const int x = __shfl_down_sync(~0u, most, d), its = __shfl_down_sync(~0u, mine, d);
            if (lane + d < 32 && its == mine) most = max(most, x);
        }
    }
    return w.base + lane < a.M && begins ? tiles_of<ROWS>(a, most) + kUnitCost : 0;
}

// 16 bytes, the first n of them from memory and zeros behind.
__device__ __forceinline__ void copy16(unsigned to, const void *from, int n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
}
__device__ __forceinline__ unsigned long long times(int a, unsigned b) { return (unsigned long long)(unsigned)a * b; }

// A piece of a unit: tiles [first, last) of `tiles`.
struct Piece {
    int i, unit, first, last, tiles;   // unit: of the token
    Pack p;
};

// The rows of a piece's tiles on their way into shared memory.  ALIGNED: pages are whole tiles, so a tile lies in one page and its rows are a stride apart;
// a lane looks up a tile, 32 at a time; else it looks up a row, the 2 (4) tiles of 32 rows at a time.  The next lot is looked up in two steps, the index in
// the table and the page, while the tiles of this one are taken.
template <typename T, int W, bool ALIGNED> struct Feed {
    using F = Form<T, W>;
    static constexpr int N = 16 / sizeof(T), CHUNKS = F::ROW / 16, PER = F::ROWS * CHUNKS / 32;   // elements of 16 bytes; of a row; copies of a lane
    static constexpr int AT_ONCE = CHUNKS > 32 ? 1 : 32 / CHUNKS;                                   // rows of a warp's copy (1024 bytes: half of one)
    static constexpr int LOT = ALIGNED ? 32 : 32 / F::ROWS;                                         // tiles
    static constexpr unsigned ALL = ~0u >> (32 - F::ROWS);
    const AttnArgs<T> &a;
    const int *table, *list;
    const char *k, *v;
    int lane, seen, n, tile, last, lot;   // n: positions of the unit's line; the next tile to copy, the piece's end; the lot's first tile
    int held, row, left;                  // of the lot: page (-1: nothing there), row of it, ALIGNED: rows that are there
    int next_index, next_row, next_held;  // of the next lot
    bool looked_up;                       // next_held is known
    int size0, size1;                     // bytes that this lane's copies take (rows of 1024 bytes: two kinds)
    unsigned place;

    __device__ __forceinline__ Feed(const AttnArgs<T> &a_, int lane_) : a(a_), lane(lane_)
    {
        const int r = lane / CHUNKS, chunk = lane % CHUNKS;
        size0 = min(max((a.d - chunk * N) * (int)sizeof(T), 0), 16);
        size1 = CHUNKS > 32 ? min(max((a.d - (lane + 32) * N) * (int)sizeof(T), 0), 16) : size0;
        // bfloat16: a row's 16-byte pieces are turned by the row, so that eight rows' pieces at one place lie in different banks
        place = r * F::ROW + (sizeof(T) == 2 ? chunk ^ r : chunk) * 16;
        tile = last = 0;
    }
    __device__ __forceinline__ void index(int first)   // of the next lot, from tile `first` on
    {
        const unsigned p = ALIGNED ? ((unsigned)first + lane) * F::ROWS : (unsigned)first * F::ROWS + lane;
        next_index = -1;
        next_row = 0;
        if (p < (unsigned)n) {
            next_index = (int)a.by_page(p);
            next_row = (int)p - next_index * a.page;
            if (list) next_index = list[next_index];
        }
        looked_up = false;
    }
    __device__ __forceinline__ void look_up()
    {
        if (looked_up) return;
        if (list && (next_index < 0 || next_index * (long long)a.page + next_row >= seen)) next_index = -1;
        next_held = next_index < 0 ? -1 : table[next_index];
        looked_up = true;
    }
    __device__ __forceinline__ void begin(const Piece &x, int request)
    {
        const int g = (int)a.by_blocks((unsigned)x.unit);
        seen = x.p.most;
        table = a.t.entries + (seen ? times(request, (unsigned)a.t.ld) : 0);
        list = a.lists ? a.lists + times(x.i * a.kv_heads + g, a.keep) : nullptr;
        n = line_of(a, seen);
        k = a.k.data + times(g, a.k.sh);
        v = a.v.data + times(g, a.v.sh);
        if (ALIGNED) {   // (what a lane does not read is not pointed to either)
            k += times(lane / CHUNKS, a.k.ld);
            v += times(lane / CHUNKS, a.v.ld);
        }
        k += size0 ? lane % CHUNKS * 16 : 0;
        v += size0 ? lane % CHUNKS * 16 : 0;
        tile = x.first;
        last = x.last;
        lot = x.first - LOT;   // (the next one begins with the piece)
        index(x.first);
    }
    __device__ __forceinline__ bool ready() const { return tile - lot < LOT || looked_up; }
    static __device__ __forceinline__ unsigned to_of(unsigned to, unsigned place, int i)   // of copy i
    {
        if (CHUNKS > 32) return to + (i / 2) * F::ROW + (i & 1) * 512 + place;
        return to + i * AT_ONCE * F::ROW + (sizeof(T) == 2 ? place ^ ((i * AT_ONCE & 7) * 16) : place);
    }
    // Begins the copies of the next tile; which of its rows are there.
    __device__ __forceinline__ unsigned copy(unsigned to)
    {
        if (tile - lot == LOT) {   // a new lot
            look_up();
            lot = tile;
            held = (unsigned)next_held < (unsigned)a.pages ? next_held : -1;
            row = next_row;
            if (ALIGNED) left = held < 0 ? 0 : min(seen - (next_index * a.page + next_row), F::ROWS);
            if (tile + LOT < last) index(tile + LOT);
        }
        const int at = tile++ - lot;
        if (ALIGNED) {
            const int rows = __shfl_sync(~0u, left, at), page = __shfl_sync(~0u, held, at), first = __shfl_sync(~0u, row, at);
            if (rows == 0) return 0;
            const char *kr = k + times(page, a.k.sp) + times(first, a.k.ld), *vr = v + times(page, a.v.sp) + times(first, a.v.ld);
            const unsigned long long k_step = (unsigned long long)a.k.ld * AT_ONCE, v_step = (unsigned long long)a.v.ld * AT_ONCE;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int r = CHUNKS > 32 ? i / 2 : i * AT_ONCE + lane / CHUNKS, half = CHUNKS > 32 ? i & 1 : 0;
                const int size = r < rows ? (half ? size1 : size0) : 0, more = half && size1 ? 512 : 0;
                copy16(to_of(to, place, i), kr + more, size);
                copy16(to_of(to, place, i) + F::ROWS * F::ROW, vr + more, size);
                if (CHUNKS <= 32 || half) { kr += k_step; vr += v_step; }
            }
            return ALL >> (F::ROWS - rows);
        } else {
            const unsigned there = __ballot_sync(~0u, held >= 0) >> (at * F::ROWS & 31) & ALL;
            if (!there) return 0;
            const unsigned long long at_k = held < 0 ? 0 : times(held, a.k.sp) + times(row, a.k.ld), at_v = held < 0 ? 0 : times(held, a.v.sp) + times(row, a.v.ld);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int r = CHUNKS > 32 ? i / 2 : i * AT_ONCE + lane / CHUNKS, half = CHUNKS > 32 ? i & 1 : 0;
                const int size = there >> r & 1 ? (half ? size1 : size0) : 0, more = half && size1 ? 512 : 0;
                copy16(to_of(to, place, i), k + __shfl_sync(~0u, at_k, at * F::ROWS + r) + more, size);
                copy16(to_of(to, place, i) + F::ROWS * F::ROW, v + __shfl_sync(~0u, at_v, at * F::ROWS + r) + more, size);
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
    __device__ __forceinline__ const T *query(int c) const { int t, h; of(c, t, h); return a.q + (times(t, a.q_ld) + times(h, a.q_sh)); }
    __device__ __forceinline__ T *out(int c) const { int t, h; of(c, t, h); return a.out + (times(t, a.out_ld) + times(h, a.out_sh)); }
    __device__ __forceinline__ float *lse(int c) const { int t, h; of(c, t, h); return a.lse + (t * a.heads + h); }
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
// A weight goes into its product as two bfloat16 that make up 16 bits of it, so that results are as far from the formula as their own rounding alone makes
// them; with one the products take a third less, which the largest case does not notice (198 instead of 203 us) and calls of short rows do (36 instead of 39).
// A weight of 0 (of a query that does not see a row which others of its unit see) or a lower part makes NaN of an infinity in V, so a unit whose sums are not
// finite is taken again, and then what is not finite goes into the sums of those that see it by itself, and not into the products.
template <int W, int NT> struct Tile16 {
    static constexpr int QUERIES = 8 * NT, KS = W / 16;
    // a unit's queries are loaded while the one before it is taken (wider ones would not fit); sixteen of the widest stay in shared memory
    static constexpr bool EARLY = W < 256, STORED = W == 256 && NT == 2;
    unsigned q[STORED ? 1 : KS][NT][2], early[EARLY ? KS : 1][NT][2];
    float o[KS][NT][4];       // [columns 16 x ..][queries 8 x ..]: columns g, g + 8 (pairs), queries 2 t, 2 t + 1
    float base[NT][2], ahead[NT][2], sum[NT][2];   // of queries 2 t, 2 t + 1; ahead: by how much a logit may exceed base (-inf: none has been met)
    int sees[NT][2];
    bool apart;               // what is not finite in V is not in the products

    static __device__ __forceinline__ void load(const Queries<Bf16> &u, int lane, unsigned (&to)[KS][NT][2])
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int m = 0; m < NT; ++m) {
            const int c = m * 8 + g;
            const Bf16 *p = u.query(c < u.n ? c : 0);
            const int d = c < u.n ? u.a.d : 0;
            if (u.a.pairs) {   // (the same for all: no branches around single loads)
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int e = s * 16 + x * 8 + t * 2;
                        to[s][m][x] = e < d ? *reinterpret_cast<const unsigned *>(p + e) : 0;
                    }
            } else {
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int e = s * 16 + x * 8 + t * 2;
                        const unsigned y = e < d ? p[e].bits : 0, z = e + 1 < d ? p[e + 1].bits : 0;
                        to[s][m][x] = y | z << 16;
                    }
            }
        }
    }
    __device__ __forceinline__ void look_ahead(const Queries<Bf16> &u, int lane) { if constexpr (EARLY) load(u, lane, early); }
    // at_once: nothing was loaded early
    __device__ __forceinline__ void begin(const Queries<Bf16> &u, int lane, bool alike, bool at_once, char *stored)
    {
        if constexpr (STORED) {
            for (int x = lane; x < QUERIES * (W / 8); x += 32) {   // (of eight neighbouring elements each)
                const int c = x / (W / 8), chunk = x % (W / 8), e = chunk * 8;
                Chunk<Bf16> y;
                y.u = make_uint4(0, 0, 0, 0);
                if (c < u.n) y.load(u.query(c), e, u.a.d, u.a.fours && e + 8 <= u.a.d);
                *reinterpret_cast<uint4 *>(stored + c * Form<Bf16, W>::ROW + (chunk ^ (c & 7)) * 16) = y.u;
            }
            __syncwarp();
        } else if (EARLY && !at_once) {
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int m = 0; m < NT; ++m) { q[s][m][0] = early[EARLY ? s : 0][m][0]; q[s][m][1] = early[EARLY ? s : 0][m][1]; }
        } else if constexpr (!STORED) {
            load(u, lane, q);
        }
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e) sees[m][e] = alike ? INT_MAX : u.sees(m * 8 + 2 * (lane & 3) + e);
        apart = false;
        clear();
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
    // there: the tile's rows that are there; first: the position of its row 0, or -1 if all queries see all of them.  APART: see `apart`.
    template <bool APART> __device__ __forceinline__ void take(char *tile, unsigned there, int first, float scale2, int lane, char *stored)
    {
        using F = Form<Bf16, W>;
        constexpr int H = F::ROWS / 16, SUMS = H == 1 ? 2 : 1;   // sixteens of rows; sums of a product (so that few products wait for one another)
        const unsigned at = (unsigned)__cvta_generic_to_shared(tile);
        float x[H][NT][4] = {};
        {
            float y[H][NT][4] = {};
            const int row = lane & 15;
            const unsigned from = at + row * F::ROW, turn = ((lane >> 4) ^ (row & 7)) * 16;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    unsigned k[4];
                    load_matrices(k, from + h * 16 * F::ROW + (turn ^ (s & 3) * 32) + (s >> 2) * 128);
                    if constexpr (STORED) {
                        unsigned b[4];
                        const int c = (lane >> 4) * 8 + (lane & 7);
                        load_matrices(b, (unsigned)__cvta_generic_to_shared(stored) + c * F::ROW + (((lane >> 3 & 1) ^ (lane & 7)) * 16 ^ (s & 3) * 32) + (s >> 2) * 128);
#pragma unroll
                        for (int m = 0; m < NT; ++m) mma_bf16(s % SUMS ? y[h][m] : x[h][m], k, b[2 * m], b[2 * m + 1]);
                    } else {
#pragma unroll
                        for (int m = 0; m < NT; ++m) mma_bf16(s % SUMS ? y[h][m] : x[h][m], k, q[s][m][0], q[s][m][1]);
                    }
                }
            if (SUMS == 2) {
#pragma unroll
                for (int m = 0; m < NT; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[0][m][e] += y[0][m][e];
            }
        }
        const int g = lane >> 2;
        bool move = false;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[h][m][e] = fmaf(x[h][m][e], scale2, -base[m][e & 1]);
        if (there != ~0u >> (32 - F::ROWS) || first >= 0) {
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int m = 0; m < NT; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int row = h * 16 + (e < 2 ? g : g + 8);
                        if (!(there >> row & 1) || (first >= 0 && first + row >= sees[m][e & 1])) x[h][m][e] = -CUDART_INF_F;
                    }
        }
        float most[NT][2];
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                most[m][e] = fmaxf(x[0][m][e], x[0][m][e + 2]);
                if (H == 2) most[m][e] = fmaxf(most[m][e], fmaxf(x[H - 1][m][e], x[H - 1][m][e + 2]));
                move |= most[m][e] > ahead[m][e];
            }
        if (__any_sync(~0u, move)) {
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float by = most[m][e];
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) by = fmaxf(by, __shfl_xor_sync(~0u, by, w));
                    float fall = 1.f;
                    if (by == -CUDART_INF_F) by = 0.f;
                    else if (ahead[m][e] == kAhead) fall = attn::ex2(-(by = fmaxf(by, 0.f)));
                    else ahead[m][e] = kAhead;   // the first logit, which may lie far below 0
                    base[m][e] += by;
#pragma unroll
                    for (int h = 0; h < H; ++h) { x[h][m][e] -= by; x[h][m][e + 2] -= by; }
                    sum[m][e] *= fall;
#pragma unroll
                    for (int s = 0; s < KS; ++s) { o[s][m][e] *= fall; o[s][m][e + 2] *= fall; }
                }
        }
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[h][m][e] = attn::ex2(x[h][m][e]);
                    sum[m][e & 1] += x[h][m][e];
                }
        if (APART) set_apart<H>(tile + F::ROWS * F::ROW, there, first, x, lane);
        unsigned high[H][NT][2], low[H][NT][2];
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int m = 0; m < NT; ++m) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const unsigned u = attn::bf16x2(x[h][m][2 * j], x[h][m][2 * j + 1]);
                    high[h][m][j] = transposed(u);
                    low[h][m][j] = transposed(attn::bf16x2(x[h][m][2 * j] - __uint_as_float(u << 16), x[h][m][2 * j + 1] - __uint_as_float(u & 0xffff0000u)));
                }
            }
        const int row = (lane >> 4) * 8 + (lane & 7);
        const unsigned from = at + (F::ROWS + row) * F::ROW, turn = ((lane >> 3 & 1) ^ (lane & 7)) * 16;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                unsigned v[4];
                load_transposed(v, from + h * 16 * F::ROW + (turn ^ (s & 3) * 32) + (s >> 2) * 128);
#pragma unroll
                for (int m = 0; m < NT; ++m) {
                    mma_bf16(o[s][m], v, high[h][m][0], high[h][m][1]);
                    mma_bf16(o[s][m], v, low[h][m][0], low[h][m][1]);
                }
            }
    }
    // A tile's values that are not finite: into the sums of the queries that see their rows, and zeros in their place.  p: the weights, as `take` has them.
    template <int H> __device__ void set_apart(char *values, unsigned there, int first, const float (&p)[H][NT][4], int lane)
    {
        using F = Form<Bf16, W>;
        const int g = lane >> 2, t = lane & 3;
#pragma unroll 1
        for (int row = 0; row < F::ROWS; ++row) {
            if (!(there >> row & 1)) continue;   // (zeros)
#pragma unroll 1
            for (int s = 0; s < 2 * KS; ++s) {
                Bf16 *at = reinterpret_cast<Bf16 *>(values + row * F::ROW + (s ^ (row & 7)) * 16) + g;
                const unsigned u = at->bits;
                const bool odd = (u & 0x7f80) == 0x7f80;
                if (!__any_sync(~0u, odd)) continue;
#pragma unroll 1
                for (int m = 0; m < NT; ++m)
#pragma unroll 1
                    for (int e = 0; e < 2; ++e) {
                        const float w = __shfl_sync(~0u, p[row >> 4][m][(row >> 3 & 1) * 2 + e], (row & 7) * 4 + t);
                        float &to = o[s >> 1][m][(s & 1) * 2 + e];
                        if (odd && (first < 0 || first + row < sees[m][e])) to = fmaf(w, __uint_as_float(u << 16), to);
                    }
                if (odd && t == 0) at->bits = 0;   // (all four lanes that look at it have read it)
            }
        }
        __syncwarp();
    }
    // True: to be taken again.  (Tile32: only where not all queries see the same)
    __device__ __forceinline__ bool again(bool)
    {
        bool odd = false;
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= !(fabsf(o[s][m][e]) <= 3.402823466e38f);
        odd = __any_sync(~0u, odd) && !apart;
        apart |= odd;
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
            const int c = m * 8 + g, d = c < u.n ? u.a.d : 0;
            Bf16 *out = u.out(c < u.n ? c : 0) + 2 * t;
            unsigned y[KS][2];   // columns by queries to queries by columns: this lane's query g, columns 2 t and 2 t + 1 of eight
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int j = 0; j < 2; ++j) y[s][j] = transposed(attn::bf16x2(o[s][m][2 * j] * f[0], o[s][m][2 * j + 1] * f[1]));
            if (u.a.pairs) {
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (s * 16 + j * 8 + 2 * t < d) *reinterpret_cast<unsigned *>(out + s * 16 + j * 8) = y[s][j];
            } else {
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int e = s * 16 + j * 8 + 2 * t;
                        if (e < d) out[s * 16 + j * 8].bits = (unsigned short)y[s][j];
                        if (e + 1 < d) out[s * 16 + j * 8 + 1].bits = (unsigned short)(y[s][j] >> 16);
                    }
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
                const bool on = c < queries;
                float *to = part + c * W + g;
                if (on && g == 0) ml[c] = make_float2(ahead[m][e] == kAhead ? base[m][e] : -CUDART_INF_F, sum[m][e]);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    if (on) to[s * 16] = o[s][m][e];
                    if (on) to[s * 16 + 8] = o[s][m][e + 2];
                }
            }
    }
};

// The same in fp32, on the CUDA cores, two sums an instruction, for Q = 4 or 8 queries.  A lane of S has a query (lane % Q) and every PARTS-th 16 bytes of it in
// registers, and reads those of each row of K along with the other queries' lanes; PARTS lanes' sums then go to one of them for each row.  A lane of
// O has W / 32 columns of all queries and reads the weights, which pass through shared memory.
template <int W, int Q> struct Tile32 {
    static constexpr int QUERIES = Q, PARTS = 32 / Q, ROWS = Form<float, W>::ROWS, MINE = ROWS / PARTS, COLS = W / 32, FOURS = W / 4 / PARTS;
    static constexpr bool EARLY = W < 128;   // as above
    uint64_t q[FOURS][2], early[EARLY ? FOURS : 1][2], o[Q / 2][COLS];   // o: pairs of queries, columns
    float base, ahead, sum;
    int sees;
    bool apart;               // as above

    static __device__ __forceinline__ void load(const Queries<float> &u, int lane, uint64_t (&to)[FOURS][2])
    {
        const int c = lane % Q, part = lane / Q;
        const float *p = u.query(c < u.n ? c : 0) + part * 4;
        const int d = c < u.n ? u.a.d - part * 4 : 0;
        if (u.a.fours) {
#pragma unroll
            for (int i = 0; i < FOURS; ++i) {
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                if (i * PARTS * 4 < d) x = *reinterpret_cast<const float4 *>(p + i * PARTS * 4);
                to[i][0] = attn::two(x.x, x.y);
                to[i][1] = attn::two(x.z, x.w);
            }
        } else {
#pragma unroll
            for (int i = 0; i < FOURS; ++i) {
                float x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = i * PARTS * 4 + k < d ? p[i * PARTS * 4 + k] : 0.f;
                to[i][0] = attn::two(x[0], x[1]);
                to[i][1] = attn::two(x[2], x[3]);
            }
        }
    }
    __device__ __forceinline__ void look_ahead(const Queries<float> &u, int lane) { if constexpr (EARLY) load(u, lane, early); }
    __device__ __forceinline__ void begin(const Queries<float> &u, int lane, bool alike, bool at_once, char *)
    {
        if (EARLY && !at_once) {
#pragma unroll
            for (int i = 0; i < FOURS; ++i) { q[i][0] = early[EARLY ? i : 0][0]; q[i][1] = early[EARLY ? i : 0][1]; }
        } else {
            load(u, lane, q);
        }
        sees = alike ? INT_MAX : u.sees(lane % Q);
        apart = false;
        clear();
    }
    __device__ __forceinline__ void clear()
    {
        ahead = -CUDART_INF_F; base = 0.f; sum = 0.f;
#pragma unroll
        for (int h = 0; h < Q / 2; ++h)
#pragma unroll
            for (int c = 0; c < COLS; ++c) o[h][c] = 0;
    }
    static __device__ __forceinline__ int weights_of(int row) { return row * Q + row / MINE * Q; }   // (rows that are written at once lie in different banks)
    template <bool APART> __device__ __forceinline__ void take(char *tile, unsigned there, int first, float scale2, int lane, char *stored)
    {
        float *weights = reinterpret_cast<float *>(stored);
        using F = Form<float, W>;
        const int part = lane / Q;
        float s[ROWS];
        const char *from = tile + part * 16;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            uint64_t x = 0, y = 0;
#pragma unroll
            for (int i = 0; i < FOURS; ++i) {
                const ulonglong2 k = *reinterpret_cast<const ulonglong2 *>(from + r * F::ROW + i * PARTS * 16);
                x = attn::fma2(q[i][0], k.x, x);
                y = attn::fma2(q[i][1], k.y, y);
            }
            float u, v;
            attn::split(attn::add2(x, y), u, v);
            s[r] = u + v;
        }
        // PARTS lanes' sums of every row -> one lane's: rows part * MINE ...
#pragma unroll
        for (int w = 16, n = ROWS / 2; w >= Q; w >>= 1, n >>= 1) {
            const bool up = lane & w;
#pragma unroll
            for (int r = 0; r < ROWS / 2; ++r)
                if (r < n) {
                    const float give = up ? s[r] : s[r + n], keep = up ? s[r + n] : s[r];
                    s[r] = keep + __shfl_xor_sync(~0u, give, w);
                }
        }
        bool move = false;
#pragma unroll
        for (int r = 0; r < MINE; ++r) {
            s[r] = fmaf(s[r], scale2, -base);
            const int row = part * MINE + r;
            if (!(there >> row & 1) || (first >= 0 && first + row >= sees)) s[r] = -CUDART_INF_F;
            move |= s[r] > ahead;
        }
        if (__any_sync(~0u, move)) {
            float by = s[0];
#pragma unroll
            for (int r = 1; r < MINE; ++r) by = fmaxf(by, s[r]);
#pragma unroll
            for (int w = Q; w < 32; w <<= 1) by = fmaxf(by, __shfl_xor_sync(~0u, by, w));
            float fall = 1.f;
            if (by == -CUDART_INF_F) by = 0.f;
            else if (ahead == kAhead) fall = attn::ex2(-(by = fmaxf(by, 0.f)));
            else ahead = kAhead;
            base += by;
            sum *= fall;
#pragma unroll
            for (int r = 0; r < MINE; ++r) s[r] -= by;
#pragma unroll
            for (int h = 0; h < Q / 2; ++h) {
                const uint64_t f = attn::two(__shfl_sync(~0u, fall, 2 * h), __shfl_sync(~0u, fall, 2 * h + 1));
#pragma unroll
                for (int c = 0; c < COLS; ++c) o[h][c] = attn::mul2(o[h][c], f);
            }
        }
#pragma unroll
        for (int r = 0; r < MINE; ++r) {
            s[r] = attn::ex2(s[r]);
            sum += s[r];
            weights[weights_of(part * MINE + r) + lane % Q] = s[r];
        }
        __syncwarp();
        if (APART) set_apart(tile + ROWS * F::ROW, there, first, weights, lane);
        const char *v_from = tile + ROWS * F::ROW + lane * (COLS == 2 ? 8 : 16);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float v[COLS];
            if constexpr (COLS == 2) {
                const float2 y = *reinterpret_cast<const float2 *>(v_from + r * F::ROW);
                v[0] = y.x; v[1] = y.y;
            } else {
#pragma unroll
                for (int c = 0; c < COLS; c += 4) {
                    const float4 y = *reinterpret_cast<const float4 *>(v_from + r * F::ROW + c * 128);
                    v[c] = y.x; v[c + 1] = y.y; v[c + 2] = y.z; v[c + 3] = y.w;
                }
            }
            uint64_t p[Q / 2];
#pragma unroll
            for (int h = 0; h < Q / 2; h += 2) {
                const ulonglong2 y = reinterpret_cast<const ulonglong2 *>(weights + weights_of(r))[h / 2];
                p[h] = y.x; p[h + 1] = y.y;
            }
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const uint64_t x = attn::two(v[c], v[c]);
#pragma unroll
                for (int h = 0; h < Q / 2; ++h) o[h][c] = attn::fma2(p[h], x, o[h][c]);
            }
        }
    }
    // As above; weights: of the tile.  A lane looks at its own columns.
    __device__ void set_apart(char *values, unsigned there, int first, const float *weights, int lane)
    {
        using F = Form<float, W>;
#pragma unroll 1
        for (int row = 0; row < ROWS; ++row) {
            if (!(there >> row & 1)) continue;
#pragma unroll 1
            for (int c = 0; c < COLS; ++c) {
                float *at = reinterpret_cast<float *>(values + row * F::ROW) + column(c, lane);
                const float v = *at;
                const bool odd = !(fabsf(v) <= 3.402823466e38f);
                if (!__any_sync(~0u, odd)) continue;
#pragma unroll 1
                for (int h = 0; h < Q / 2; ++h) {
                    const bool see0 = first < 0 || first + row < __shfl_sync(~0u, sees, 2 * h), see1 = first < 0 || first + row < __shfl_sync(~0u, sees, 2 * h + 1);
                    float x, y;
                    attn::split(o[h][c], x, y);
                    if (odd && see0) x = fmaf(weights[weights_of(row) + 2 * h], v, x);
                    if (odd && see1) y = fmaf(weights[weights_of(row) + 2 * h + 1], v, y);
                    o[h][c] = attn::two(x, y);
                }
                if (odd) *at = 0.f;
            }
        }
    }
    // (a weight of 0 that is not one of a row unseen is the formula's own)
    __device__ __forceinline__ bool again(bool uneven)
    {
        if (!uneven || apart) return false;
        bool odd = false;
#pragma unroll
        for (int h = 0; h < Q / 2; ++h)
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                float x, y;
                attn::split(o[h][c], x, y);
                odd |= !(fabsf(x) <= 3.402823466e38f) || !(fabsf(y) <= 3.402823466e38f);
            }
        return apart = __any_sync(~0u, odd);
    }
    __device__ __forceinline__ void total()
    {
#pragma unroll
        for (int w = Q; w < 32; w <<= 1) sum += __shfl_xor_sync(~0u, sum, w);
    }
    static __device__ __forceinline__ int column(int c, int lane) { return COLS == 2 ? lane * 2 + c : lane * 4 + c / 4 * 128 + c % 4; }
    __device__ __forceinline__ void write(const Queries<float> &u, int lane)
    {
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        if (lane < u.n) *u.lse(lane) = lse_of(base, sum);
#pragma unroll
        for (int h = 0; h < Q / 2; ++h) {
            if (2 * h >= u.n) break;
            const float f0 = __shfl_sync(~0u, f, 2 * h), f1 = __shfl_sync(~0u, f, 2 * h + 1);
            float *out0 = u.out(2 * h), *out1 = u.out(min(2 * h + 1, u.n - 1));
            const int d0 = u.a.d, d1 = 2 * h + 1 < u.n ? d0 : 0;
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const int e = column(c, lane);
                float x, y;
                attn::split(o[h][c], x, y);
                if (e < d0) out0[e] = x * f0;
                if (e < d1) out1[e] = y * f1;
            }
        }
    }
    __device__ __forceinline__ void leave(float *part, float2 *ml, int queries, int lane)
    {
        if (lane < queries) ml[lane] = make_float2(ahead == kAhead ? base : -CUDART_INF_F, sum);
#pragma unroll
        for (int h = 0; h < Q / 2; ++h)
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                float x, y;
                attn::split(o[h][c], x, y);
                if (2 * h < queries) part[2 * h * W + column(c, lane)] = x;
                if (2 * h + 1 < queries) part[(2 * h + 1) * W + column(c, lane)] = y;
            }
    }
};
// A tile on the second pass over a unit.  (Out of line and on a copy, so that what hardly any unit needs is not among the instructions and registers of all: in line
// fp32 with 64 heads over 4 took 242 instead of 223 us.)
template <typename Tile> __device__ __noinline__ void take_apart(Tile &x, char *tile, unsigned there, int first, float scale2, int lane, char *stored)
{
    x.template take<true>(tile, there, first, scale2, lane, stored);
}
template <typename T, int W, int Q> struct TileOf { using type = Tile16<W, Q / 8>; };
template <int W, int Q> struct TileOf<float, W, Q> { using type = Tile32<W, Q>; };

// The warp's pieces follow one another without a pause: while one is taken, the rows of the next one are looked up and copied and its queries loaded.
template <typename T, int W, int Q, bool ALIGNED>
__global__ void __launch_bounds__(kAttnWarps * 32, Form<T, W, Q>::CTAS) paged_attention_kernel(const AttnArgs<T> a)
{
    using F = Form<T, W, Q>;
    using Tile = typename TileOf<T, W, Q>::type;
    extern __shared__ __align__(128) char shared[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, me = blockIdx.x * kAttnWarps + warp;
    const int units = a.kv_heads * a.blocks;   // of a token
    char *ring = shared + warp * F::RING;
    const unsigned ring_at = (unsigned)__cvta_generic_to_shared(ring);
    char *stored = shared + kAttnWarps * F::RING + warp * F::STORED;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
    Share share;
    Window window;
    const auto load = [&](int base) { return window_of(a, base, lane); };
    const auto cost = [&](const Window &w) { return cost_of<F::ROWS>(a, window = w, lane); };
    if (!deal<kAttnWarps * 32>(a.M, units, load, cost, gridDim.x * kAttnWarps, me, kLeastCost, share)) {
        if (!a.by_unit && lane == 0) a.joins[me] = make_int4(0, -1, 0, 0);
        return;
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (the joining CTAs wait for the end of this launch)
    int4 join = make_int4(0, -1, 0, 0);
    const float scale2 = a.scale * attn::kLog2e;

    // Where the next piece begins: `at` behind the share's begin, `before` behind the begin of a unit; tile t of the unit lies at kUnitCost + t.
    Pack pack = pack_of(a, window, share.row, lane);
    int token = share.row, tiles = tiles_of<F::ROWS>(a, pack.most), unit = (int)quotient(share.rest, tiles + kUnitCost);
    const int size = (int)(share.hi - share.lo);   // (of 2^27 tiles of a row and 2^31 rows at most, in shares of thousands of them)
    int at = 0, before = (int)(share.rest - (long long)unit * (tiles + kUnitCost));
    const auto queries_of = [&](const Piece &x) {
        const int g = (int)a.by_blocks((unsigned)x.unit), b = x.unit - g * a.blocks;
        return Queries<T>{a, x.i, g * a.group + b * Tile::QUERIES, a.pack > 1 ? x.p.n * a.group : min(Tile::QUERIES, a.group - b * Tile::QUERIES)};
    };
    Feed<T, W, ALIGNED> feed(a, lane);
    Tile x;
    const auto next_piece = [&](Piece &to) {   // false: there is none
        while (at < size) {
            const int begin = at - before, end = min(begin + tiles + kUnitCost, size);
            to.i = token; to.unit = unit; to.tiles = tiles; to.p = pack;
            to.first = max(before - kUnitCost, 0);
            to.last = end - begin - kUnitCost;
            // a unit that begins here and ends elsewhere: its last tile lies with the last warp
            if (to.first == 0 && to.last > 0 && to.last < tiles)
                join = make_int4(token * units + unit, me, me + (int)((unsigned)(begin + tiles + kUnitCost - 1) / (unsigned)share.share), 0);
            at = end;
            before = 0;
            if (++unit == units) {
                unit = 0;
                token += pack.n;
                if (at < size && token < a.M) {
                    if (token >= window.base + 32) window = window_of(a, token & ~31, lane);
                    pack = pack_of(a, window, token, lane);
                    tiles = tiles_of<F::ROWS>(a, pack.most);
                }
            }
            if (to.last > to.first) return true;
            if (token >= a.M) return false;   // (not with lengths that stay as they are)
        }
        return false;
    };
    const auto start = [&](const Piece &p) { feed.begin(p, p.p.most ? row_of(a.tok, p.i) : 0); };   // its rows
    Piece now, next;
    if (!next_piece(now)) {
        if (!a.by_unit && lane == 0) a.joins[me] = join;
        return;
    }
    start(now);
    bool more = false, fed = false;   // there is a next piece; its rows are being copied
    x.begin(queries_of(now), lane, now.p.n == 1, true, stored);
    int ahead = 0, stage = 0, j = now.first;   // tiles that are on their way; the stage of the oldest, the tile that it is
    unsigned there0 = 0, there1 = 0, there2 = 0;
    for (;;) {
        while (ahead < kStages && feed.tile < feed.last && (ahead < 2 || feed.ready())) {
            const int to = stage + ahead;
            const unsigned there = feed.copy(ring_at + (to >= kStages ? to - kStages : to) * F::TILE);
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (ahead == 0) there0 = there; else if (ahead == 1) there1 = there; else there2 = there;
            ++ahead;
        }
        if (ahead == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (ahead == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        if (there0) {
            char *tile = ring + stage * F::TILE;
            const int first = now.p.n > 1 && j * F::ROWS > now.p.least - F::ROWS ? j * F::ROWS : -1;   // (the end of a row's last tile may lie at 2^31)
            if (__builtin_expect(!x.apart, 1)) {
                x.template take<false>(tile, there0, first, scale2, lane, stored);
            } else {
                Tile y = x;
                take_apart(y, tile, there0, first, scale2, lane, stored);
                x = y;
            }
        }
        there0 = there1;
        there1 = there2;
        --ahead;
        stage = stage == kStages - 1 ? 0 : stage + 1;
        feed.look_up();
        __syncwarp();
        if (feed.tile == feed.last && !fed) {   // all of this piece is on its way: the next one
            if (!more) more = next_piece(next);
            if (more) { start(next); fed = true; x.look_ahead(queries_of(next), lane); }
        }
        if (++j < now.last) continue;
        if (x.again(now.p.least < now.p.most)) {   // from its first tile on, without what is on its way of the next
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
            x.clear();
            ahead = 0;
            fed = false;
            j = now.first;
            start(now);
            continue;
        }
        x.total();
        const int id = now.i * units + now.unit;
        const bool all = now.first == 0 && now.last == now.tiles;
        const Queries<T> u = queries_of(now);
        if (all) {
            x.write(u, lane);
        } else {
            const long long slot = me * 2ll + (now.first == 0);
            x.leave(a.part + slot * Tile::QUERIES * W, a.part_ml + slot * Tile::QUERIES, u.n, lane);
            if (now.first == 0) join.w = u.n;
        }
        if (now.first == 0 && a.by_unit && lane < now.p.n) a.joins[id + lane * units] = lane == 0 && !all ? join : make_int4(0, -1, 0, 0);
        if (!more) break;
        now = next;
        more = fed = false;
        j = now.first;
        x.begin(queries_of(now), lane, now.p.n == 1, false, stored);
    }
    if (!a.by_unit && lane == 0) a.joins[me] = join;
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
