// Attention over the tiles of a plan on the tensor cores, fp32 operands, head widths up to 128.
//
// Every operand is split into three bfloat16 planes, x = x1 + x2 + x3 exactly (8 + 8 + 8 significant bits; a plane is what is left of x
// rounded to nearest), and a product is six products of planes, smallest first: x2 y2, x1 y3, x3 y1, x1 y2, x2 y1, x1 y1.  What is left out is below
// 2^-23 of each term (three times half steps of 2^-8 - 16).  The weights p and p (dp - delta) are split in the same way, in registers.
// The tensor core adds into its fp32 accumulators with truncation, about -2e-8 of the sum each time, so sums in it stay short: S and dP are
// begun with the small products, and the second products of every step start from zero and are added up in registers, rounded to nearest.
//
// What bounds it is the tensor core, six times the products of the bfloat16 kernels: two batches of 2 x 4 x 128 x 64 x 64 x 6 multiplications a
// tile forward, seven backward.  1501 x 2903, six heads of width 50 at 12% (1656 tiles): forward 61 us (of it the tiles 46), backward 180 us
// (dQ 71, dK and dV 107, side by side with what stands ahead and behind); the row kernels take 265 and 818 us.  A tile costs the same at any density: see prefer_tiles.
// Above width 64 the planes of Q, dO and a step of K and V would take 294 KB of shared memory: there the products of all tiles are computed ahead.
//
// The walk over shares of tiles, the roles and the barriers are those of tile_grad_kernel (attention_tiles.cuh).
#pragma once
#include "attention_tiles.cuh"

namespace b2sp {
namespace attn {

constexpr int kPlane = 64, kPlanes = 192;   // columns of a plane and of a row of planes in memory
constexpr int kPairs = 6;
__host__ __device__ constexpr int pair_a(int p) { return p == 0 ? 1 : p == 1 ? 0 : p == 2 ? 2 : p == 3 ? 0 : p == 4 ? 1 : 0; }
__host__ __device__ constexpr int pair_b(int p) { return p == 0 ? 1 : p == 1 ? 2 : p == 2 ? 0 : p == 3 ? 1 : p == 4 ? 0 : 0; }

// Two numbers as three planes of two bfloat16.
__device__ __forceinline__ void split3(float a, float b, uint32_t &p1, uint32_t &p2, uint32_t &p3)
{
    p1 = bf16x2(a, b);
    a -= __uint_as_float(p1 << 16);
    b -= __uint_as_float(p1 & 0xffff0000u);
    p2 = bf16x2(a, b);
    a -= __uint_as_float(p2 << 16);
    b -= __uint_as_float(p2 & 0xffff0000u);
    p3 = bf16x2(a, b);
}

// ---- operands to planes --------------------------------------------------------------------------------------------------------------
struct SplitArgs {
    View<const float> x[4];
    Bf16 *planes[4];         // [batch][heads][rows][chunks][192]
    int heads[4], rows[4], count, d, batch, chunks;
    long long before[5];     // rows of the tensors ahead
};
// Sixteen threads per row and chunk of 64 columns, four elements each; in the first CTAs, where the shares begin.
template <int V>
__global__ void __launch_bounds__(256) split_planes_kernel(const __grid_constant__ SplitArgs a, const __grid_constant__ ShareArgsOf<float> h, int share_blocks, int *status)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
    if ((int)blockIdx.x < share_blocks) {
        prepare_shares(h, a.d, share_blocks);
        return;
    }
    const int lanes = 16 * a.chunks;   // 16 or 32
    const long long row = (blockIdx.x - share_blocks) * (256ll / lanes) + threadIdx.x / lanes;
    if (row >= a.before[a.count]) return;
    int t = 0;
    while (t + 1 < a.count && row >= a.before[t + 1]) ++t;
    const long long in = row - a.before[t];
    const int prob = (int)(in / a.rows[t]), c = threadIdx.x % lanes * 4;
    float x[4];
    load4<float, V>(a.x[t].at(prob / a.heads[t], prob % a.heads[t], in % a.rows[t]), c, a.d, x);
    uint2 p[3];
    split3(x[0], x[1], p[0].x, p[1].x, p[2].x);
    split3(x[2], x[3], p[0].y, p[1].y, p[2].y);
    uint2 *to = reinterpret_cast<uint2 *>(a.planes[t] + (in * a.chunks + c / kPlane) * kPlanes + c % kPlane);
#pragma unroll
    for (int k = 0; k < 3; ++k) to[k * (kPlane / 4)] = p[k];
}

template <int ROWS> __device__ __forceinline__ void load_planes(uint32_t dst, const CUtensorMap *tm, uint32_t bar, int chunk, int row, int h, int b)
{
#pragma unroll
    for (int p = 0; p < 3; ++p) tma_load_4d(dst + p * ROWS * 128, tm, bar, chunk * kPlanes + p * kPlane, row, h, b);
}
// D = A B^T over 64 columns of planes, A 128 rows, B N rows.
template <int N> __device__ __forceinline__ void product_columns32(uint32_t d, uint32_t a, uint32_t b, int ks)
{
#pragma unroll
    for (int p = 0; p < kPairs; ++p)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < ks) mma_ss(d, a + pair_a(p) * (128 * 128 >> 4) + column_step<128>(k), b + pair_b(p) * (N * 128 >> 4) + column_step<N>(k), idesc_bf16(N, false), p > 0 || k > 0);
}
// D = A B, A's planes in tensor memory (place(plane, step of 16): columns behind `a`), B 64 rows of planes.
template <class F> __device__ __forceinline__ void product_rows32(uint32_t d, uint32_t a, uint32_t b, F place)
{
#pragma unroll
    for (int p = 0; p < kPairs; ++p)
#pragma unroll
        for (int k = 0; k < 4; ++k) mma_ts(d, a + place(pair_a(p), k), b + pair_b(p) * (64 * 128 >> 4) + row_step(k), idesc_bf16(64, true), p > 0 || k > 0);
}

constexpr int kPlaneTile = 3 * 128 * 128, kPlaneHalf = 3 * 64 * 128;   // bytes of 128 and of 64 rows of planes

struct Args32 {
    GradArgsOf<float> g;
    float2 *part_ml;     // forward
    int wide;            // outputs: rows are aligned groups of four elements
    // Widths above 64: products of tile_product32_kernel, and the 64 columns at hand
    Tiles rows;          // tiles in row order, for their numbers
    float *scores[2];    // S, and (backward) dP, of a tile: [128 keys][128 queries]
    int col0, dc;        // first column of the outputs' chunk, its width; 0 and d up to 64
};
constexpr int kScores = kTile * kTile;
// Into L2, `bytes` from `p` on (multiples of 16).
__device__ __forceinline__ void prefetch(const void *p, uint32_t bytes)
{
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(reinterpret_cast<uint64_t>(p)), "r"(bytes) : "memory");
}
// The number of tile t of the pattern of problem o = (sequence, head).
__device__ __forceinline__ long long tile_number(const Tiles &rows, int o, int t) { return rows.base(o) + t - rows.at(rows.pattern(o, 0), 0); }

// ---- products of two operands over all tiles, widths 65 to 128 --------------------------------------------------------------------------
// With rows of two chunks of 64 columns the operands of all products do not fit the shared memory of an SM, so S (and dP) of the tiles are
// computed ahead, 64 KB a tile, and the kernels below read them, once per chunk of the outputs' columns.  Sets of four warps take alternate steps of
// 64 keys out of tensor memory.  2048 tiles of width 128: 60 us for S and for dP each (tensor core 37, 134 MB written), then per chunk the forward pass
// 78 us and its join, dQ 96 and dK with dV 175 us and their join.  A query's neighbours lie side by side (score reads of the forward pass and dQ, writes); with
// eight queries side by side and then the keys dK and dV take 164 us, dQ 100, the forward pass 87.
struct Prod32 {
    static constexpr int SETS = 3, THREADS = 128 * SETS + 64, STAGES = 2, X = 0, Y = 2 * kPlaneTile, BAR = Y + STAGES * 2 * kPlaneHalf, BYTES = BAR + 512 + 1024;
    static constexpr uint32_t SET = 128, COLS = 512;   // of a set: the sums of either chunk, added up in registers (the tensor core truncates)
};
static_assert(Prod32::BYTES <= 232448, "shared memory");

__global__ void __launch_bounds__(Prod32::THREADS, 1)
tile_product32_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_y, const __grid_constant__ Args32 f, float *scores)
{
    using C = Prod32;
    constexpr int SETS = C::SETS, TMA_WARP = 4 * SETS, FIRST_WARP = TMA_WARP + 1;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (ptx::smem_u32(raw) + 1023u) & ~1023u, bars = base + C::BAR;
    auto full = [&](int s) { return bars + 8u * s; };
    auto free_ = [&](int s) { return bars + 64u + 8u * s; };
    auto s_full = [&](int w) { return bars + 128u + 8u * w; };
    auto s_free = [&](int w) { return bars + 176u + 8u * w; };
    auto flags = [&](int s) { return bars + 320u + 4u * s; };
    const uint32_t x_full = bars + 200, x_free = bars + 208, slot = bars + 232;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const GradArgsOf<float> &g = f.g;
    const TileArgsOf<float> &a = g.a;
    const Shape &s = a.g.s;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) { ptx::mbar_init(full(i), 1); ptx::mbar_init(free_(i), 1); }
        for (int i = 0; i < SETS; ++i) { ptx::mbar_init(s_full(i), 1); ptx::mbar_init(s_free(i), 4); }
        ptx::mbar_init(x_full, 1); ptx::mbar_init(x_free, 1);
        ptx::mbar_init(slot + 16, 1);   // the last products
        ptx::fence_mbar_init();
    }
    if (warp == FIRST_WARP) { ptx::tmem_alloc(slot, C::COLS); ptx::tmem_relinquish(); }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    asm volatile("griddepcontrol.wait;" ::: "memory");   // planes and shares
    const uint32_t tmem = ptx::lds32(slot);
    const int tiles = (int)(g.first[blockIdx.x + 1] - g.first[blockIdx.x]), steps = 2 * tiles;
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !wait_for(bar, parity)) { ok = false; *a.status = B2SP_ERR_TIMEOUT; }
        return ok;
    };
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return ok = __all_sync(~0u, wait(bar, parity)); };
    if (warp == TMA_WARP) {
        Walk w;
        w.start(g.w, g.starts[blockIdx.x], tiles);
        int i = 0, blocks = 0;
        for (bool more = tiles > 0; more && ok;) {
            const int b = w.o / g.w.outer, h = w.o % g.w.outer, hkv = h / (s.heads / s.kv_heads), blk = w.blk, r0 = g.tile_at[w.t] * kTile;
            const bool fresh = w.fresh, last = w.next(g.w);
            more = w.left > 0;
            if (fresh) {
                if (!wait_all(x_free, (blocks & 1) ^ 1)) break;
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(x_full, 2 * kPlaneTile);
                    for (int c = 0; c < 2; ++c) load_planes<128>(base + C::X + c * kPlaneTile, &tm_x, x_full, c, blk * kTile, h, b);
                }
                __syncwarp();
                ++blocks;
            }
            for (int half = 0; half < 2; ++half, ++i) {
                const int st = i % C::STAGES, at = r0 + half * 64;
                if (!wait_all(free_(st), (i / C::STAGES & 1) ^ 1)) break;
                if (ptx::elect_one()) {
                    ptx::sts32(flags(st), (fresh && !half ? kStepFirst : 0) | (last && half ? kStepLast : 0));
                    ptx::mbar_arrive_expect_tx(full(st), 2 * kPlaneHalf);
                    for (int c = 0; c < 2; ++c) load_planes<64>(base + C::Y + (2 * st + c) * kPlaneHalf, &tm_y, full(st), c, at, hkv, b);
                }
                __syncwarp();
            }
        }
        // copies in flight land before the CTA ends, also where another warp gave up a wait
        if (blocks) ptx::mbar_wait(x_full, (blocks - 1) & 1);
        for (int k = max(0, i - C::STAGES); k < i; ++k) ptx::mbar_wait(full(k % C::STAGES), k / C::STAGES & 1);
    } else if (warp == FIRST_WARP) {
        if (ptx::elect_one()) {
            const int ks = (s.d - kPlane + 15) >> 4;   // of the second chunk
            const uint32_t x = desc_columns(base + C::X), y0 = desc_columns(base + C::Y);
            int st = 0, ph = 0, set = 0, round = 0, blocks = 0;
            for (int i = 0; i < steps; ++i) {
                if (!wait(full(st), ph)) break;
                const uint32_t fl = ptx::lds32(flags(st));
                if ((fl & kStepFirst) && !wait(x_full, blocks++ & 1)) break;
                if (round && !wait(s_free(set), (round - 1) & 1)) break;
                ptx::tc_fence_after_sync();
                const uint32_t to = tmem + set * C::SET, y = y0 + st * (2 * kPlaneHalf >> 4);
                product_columns32<64>(to, x, y, 4);
                product_columns32<64>(to + 64, x + (kPlaneTile >> 4), y + (kPlaneHalf >> 4), ks);
                ptx::mma_commit(s_full(set));
                ptx::mma_commit(free_(st));
                if (fl & kStepLast) ptx::mma_commit(x_free);
                if (++st == C::STAGES) { st = 0; ph ^= 1; }
                if (++set == SETS) { set = 0; ++round; }
            }
            ptx::mma_commit(slot + 16);   // products in flight end before tensor memory is freed, also where another warp gave up a wait
            ptx::mbar_wait(slot + 16, 0);
        }
        __syncwarp();
    } else {
        const int set = warp >> 2, lane_row = threadIdx.x & 127;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16) + set * C::SET;
        const long long n0 = g.first[blockIdx.x];
        for (int i = set, round = 0; i < steps && ok; i += SETS, ++round) {
            if (!wait_all(s_full(set), round & 1)) break;
            ptx::tc_fence_after_sync();
            float *to = scores + (n0 + (i >> 1)) * kScores + (i & 1) * (64 * kTile) + lane_row;
#pragma unroll
            for (int c = 0; c < 64; c += 16) {
                uint32_t x[16], y[16];
                ptx::tmem_ld_32x16(mine + c, x);
                ptx::tmem_ld_32x16(mine + 64 + c, y);
                ptx::tmem_ld_wait();
                settle(x);
                settle(y);
#pragma unroll
                for (int k = 0; k < 16; ++k) to[(c + k) * kTile] = __uint_as_float(x[k]) + __uint_as_float(y[k]);
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(s_free(set));
        }
    }
    __syncwarp();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == FIRST_WARP) { ptx::tc_fence_after_sync(); ptx::tmem_dealloc(tmem, C::COLS); }
}
// Where the sums that CTA c leaves of a block lie, forward: pairs (c, block) ascend together, so c + block is theirs alone.
__device__ __forceinline__ long long part_of(int c, long long block, int set, int sets) { return (c + block) * sets + set; }

// ---- forward ---------------------------------------------------------------------------------------------------------------------
// Three sets of four softmax warps take alternate steps of 64 keys, each with a softmax of its own (reference, sum, output), which the joining
// kernel merges; so a set waits for nobody between its steps.  The reference is the largest stored product: all products of a step are compared
// with it first, which spares the mask, and those of the entries only where one of them exceeds it by 2^8 (8 heads of 4096, width 128, 30%: 820 -> 751 us,
// with less spilled, against a reference of all products; the mask in every comparison 908).  READ: S comes from memory (see tile_product32_kernel), and O has the columns of a chunk.
struct Fwd32 {
    static constexpr int SETS = 3, THREADS = 128 * SETS + 96, STAGES = 3;
    static constexpr int Q = 0, K = kPlaneTile, V = K + STAGES * kPlaneHalf, BAR = V + STAGES * kPlaneHalf, BYTES = BAR + 512 + 1024;
    static constexpr uint32_t SET = 160, COL_P3 = 64, COL_O = 96, COLS = 512;   // of a set: S (planes 1 and 2 over it), plane 3, O
};
static_assert(Fwd32::BYTES <= 232448, "shared memory");

template <bool READ>
__global__ void __launch_bounds__(Fwd32::THREADS, 1)
tile_forward32_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                      const __grid_constant__ Args32 f)
{
    using C = Fwd32;
    constexpr int SETS = C::SETS, TMA_WARP = 4 * SETS, FIRST_WARP = TMA_WARP + 1, SECOND_WARP = TMA_WARP + 2;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (ptx::smem_u32(raw) + 1023u) & ~1023u, bars = base + C::BAR;
    auto full = [&](int s) { return bars + 8u * s; };
    auto free_ = [&](int s) { return bars + 64u + 8u * s; };
    auto s_full = [&](int w) { return bars + 128u + 8u * w; };
    auto p_full = [&](int w) { return bars + 152u + 8u * w; };
    auto s_free = [&](int w) { return bars + 176u + 8u * w; };
    auto flags = [&](int s) { return bars + 320u + 4u * s; };
    const uint32_t x_full = bars + 200, x_free = bars + 208, slot = bars + 232;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const GradArgsOf<float> &g = f.g;
    const TileArgsOf<float> &a = g.a;
    const Shape &s = a.g.s;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) { ptx::mbar_init(full(i), 1); ptx::mbar_init(free_(i), 1); }
        for (int i = 0; i < SETS; ++i) { ptx::mbar_init(s_full(i), 1); ptx::mbar_init(p_full(i), 4); ptx::mbar_init(s_free(i), 1); }
        ptx::mbar_init(x_full, 1); ptx::mbar_init(x_free, 1);
        ptx::mbar_init(slot + 16, 1); ptx::mbar_init(slot + 24, 1);   // the last products
        ptx::fence_mbar_init();
    }
    if (warp == FIRST_WARP) { ptx::tmem_alloc(slot, C::COLS); ptx::tmem_relinquish(); }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    asm volatile("griddepcontrol.wait;" ::: "memory");   // planes and shares
    const uint32_t tmem = ptx::lds32(slot);
    const int tiles = (int)(g.first[blockIdx.x + 1] - g.first[blockIdx.x]), steps = 2 * tiles;
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !wait_for(bar, parity)) { ok = false; *a.status = B2SP_ERR_TIMEOUT; }
        return ok;
    };
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return ok = __all_sync(~0u, wait(bar, parity)); };
    if (warp == TMA_WARP) {
        Walk w;
        w.start(g.w, g.starts[blockIdx.x], tiles);
        int i = 0, blocks = 0;
        for (bool more = tiles > 0; more && ok;) {
            const int b = w.o / g.w.outer, h = w.o % g.w.outer, hkv = h / (s.heads / s.kv_heads), blk = w.blk, r0 = g.tile_at[w.t] * kTile;
            if (READ) {
                const float *at = f.scores[0] + tile_number(g.w, w.o, w.t) * kScores;
                if (ptx::elect_one()) prefetch(at, kScores * 4);
                __syncwarp();
            }
            const bool fresh = w.fresh, last = w.next(g.w);
            more = w.left > 0;
            if (!READ && fresh) {
                if (!wait_all(x_free, (blocks & 1) ^ 1)) break;
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(x_full, kPlaneTile);
                    load_planes<128>(base + C::Q, &tm_q, x_full, 0, blk * kTile, h, b);
                }
                __syncwarp();
                ++blocks;
            }
            for (int half = 0; half < 2; ++half, ++i) {
                const int st = i % C::STAGES, at = r0 + half * 64;
                if (!wait_all(free_(st), (i / C::STAGES & 1) ^ 1)) break;
                if (ptx::elect_one()) {
                    ptx::sts32(flags(st), (fresh && !half ? kStepFirst : 0) | (last && half ? kStepLast : 0));
                    ptx::mbar_arrive_expect_tx(full(st), (READ ? 1 : 2) * kPlaneHalf);
                    if (!READ) load_planes<64>(base + C::K + st * kPlaneHalf, &tm_k, full(st), 0, at, hkv, b);
                    load_planes<64>(base + C::V + st * kPlaneHalf, &tm_v, full(st), f.col0 / kPlane, at, hkv, b);
                }
                __syncwarp();
            }
        }
        // copies in flight land before the CTA ends, also where another warp gave up a wait
        if (blocks) ptx::mbar_wait(x_full, (blocks - 1) & 1);
        for (int k = max(0, i - C::STAGES); k < i; ++k) ptx::mbar_wait(full(k % C::STAGES), k / C::STAGES & 1);
    } else if (warp == FIRST_WARP) {
        if (!READ && ptx::elect_one()) {
            const int ks = (s.d + 15) >> 4;
            const uint32_t q = desc_columns(base + C::Q), k0 = desc_columns(base + C::K);
            int st = 0, ph = 0, set = 0, round = 0, blocks = 0;
            for (int i = 0; i < steps; ++i) {
                if (!wait(full(st), ph)) break;
                const uint32_t fl = ptx::lds32(flags(st));
                if ((fl & kStepFirst) && !wait(x_full, blocks++ & 1)) break;
                if (round && !wait(s_free(set), (round - 1) & 1)) break;
                product_columns32<64>(tmem + set * C::SET, q, k0 + st * (kPlaneHalf >> 4), ks);
                ptx::mma_commit(s_full(set));
                if (fl & kStepLast) ptx::mma_commit(x_free);
                if (++st == C::STAGES) { st = 0; ph ^= 1; }
                if (++set == SETS) { set = 0; ++round; }
            }
            ptx::mma_commit(slot + 16);   // products in flight end before tensor memory is freed, also where another warp gave up a wait
            ptx::mbar_wait(slot + 16, 0);
        }
        __syncwarp();
    } else if (warp == SECOND_WARP) {
        if (ptx::elect_one()) {
            const uint32_t v0 = desc_rows<64>(base + C::V);
            int st = 0, ph = 0, set = 0, round = 0;
            for (int i = 0; i < steps; ++i) {
                if (!wait(full(st), ph) || !wait(p_full(set), round & 1)) break;
                ptx::tc_fence_after_sync();
                const uint32_t at = tmem + set * C::SET;
                product_rows32(at + C::COL_O, at, v0 + st * (kPlaneHalf >> 4), [](int p, int k) { return p == 2 ? (int)C::COL_P3 + 8 * k : 16 * k + 8 * p; });
                ptx::mma_commit(s_free(set));
                ptx::mma_commit(free_(st));
                if (++st == C::STAGES) { st = 0; ph ^= 1; }
                if (++set == SETS) { set = 0; ++round; }
            }
            ptx::mma_commit(slot + 24);   // products in flight end before tensor memory is freed, also where another warp gave up a wait
            ptx::mbar_wait(slot + 24, 0);
        }
        __syncwarp();
    } else {
        const int set = warp >> 2, lane_row = threadIdx.x & 127;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16) + set * C::SET;
        const float c2 = s.scale * kLog2e;
        const uint64_t f2 = two(c2, c2);
        Walk w;
        w.start(g.w, g.starts[blockIdx.x], tiles);
        int at_set = 0, round = 0, last_turn = 0;
        bool pending = false;
        float ref = -CUDART_INF_F, acc[64];   // ref: the largest stored product of this set's steps of the block, or less by 2^8 at most
        uint64_t sums = two(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 64; ++k) acc[k] = 0.f;
        auto collect = [&] {   // the last step's O
#pragma unroll
            for (int c = 0; c < 64; c += 16) {
                uint32_t x[16];
                ptx::tmem_ld_32x16(mine + C::COL_O + c, x);
                ptx::tmem_ld_wait();
                settle(x);
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[c + k] += __uint_as_float(x[k]);
            }
        };
        for (bool more = tiles > 0; more && ok;) {
            const int blk = w.blk, o = w.o;
            const uint4 now = __ldg(a.plan.masks + (long long)w.t * kTile + lane_row);
            for (int half = 0; half < 2; ++half) {
                const bool my_turn = at_set == set;
                const int turn = round;
                if (++at_set == SETS) { at_set = 0; ++round; }
                if (!my_turn) continue;
                // (S of this step came behind the set's last product; read from memory it did not)
                if (READ ? turn && !wait_all(s_free(set), (turn - 1) & 1) : !wait_all(s_full(set), turn & 1)) break;
                ptx::tc_fence_after_sync();
                if (pending) collect();
                const float *from = READ ? f.scores[0] + tile_number(g.w, o, w.t) * kScores + half * (64 * kTile) + lane_row : nullptr;
                auto load = [&](int c, uint32_t (&x)[16]) {
                    if (READ) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(from[(c + k) * kTile]);
                        settle(x);   // (all sixteen in flight)
                    } else {
                        ptx::tmem_ld_32x16(mine + c, x);
                        ptx::tmem_ld_wait();
                        settle(x);
                    }
                };
                float top4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                for (int c = 0; c < 64; c += 16) {
                    uint32_t x[16];
                    load(c, x);
#pragma unroll
                    for (int k = 0; k < 16; k += 2) top4[k >> 1 & 3] = fmaxf(top4[k >> 1 & 3], fmaxf(__uint_as_float(x[k]), __uint_as_float(x[k + 1])));
                }
                const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
                const uint32_t w0 = half ? now.z : now.x, w1 = half ? now.w : now.y;
                if (__any_sync(~0u, (w0 | w1) && (top - ref) * c2 > 8.f)) {   // (infinity: the first entries)
                    float most = -CUDART_INF_F;   // of the stored products
#pragma unroll 1
                    for (int c = 0; c < 64; c += 16) {
                        uint32_t x[16];
                        load(c, x);
                        const uint32_t m = (c & 32 ? w1 : w0) >> (c & 16);
#pragma unroll
                        for (int k = 0; k < 16; ++k) most = fmaxf(most, m >> k & 1 ? __uint_as_float(x[k]) : -CUDART_INF_F);
                    }
                    const bool move = (most - ref) * c2 > 8.f;
                    if (__any_sync(~0u, move)) {
                        const float fall = move ? ex2((ref - most) * c2) : 1.f;
                        if (move) ref = most;
                        sums = mul2(sums, two(fall, fall));
#pragma unroll
                        for (int k = 0; k < 64; ++k) acc[k] *= fall;
                    }
                }
                const uint64_t r2 = two(-ref * c2, -ref * c2);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t x[16], p1[8], p2[8], p3[8];
                    load(16 * c, x);
                    const uint32_t m = (half ? (c & 2 ? now.w : now.z) : (c & 2 ? now.y : now.x)) >> (16 * (c & 1));
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        float y0, y1;
                        split(fma2(two(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), f2, r2), y0, y1);
                        y0 = m >> k & 1 ? ex2(y0) : 0.f;
                        y1 = m >> (k + 1) & 1 ? ex2(y1) : 0.f;
                        sums = add2(sums, two(y0, y1));
                        split3(y0, y1, p1[k >> 1], p2[k >> 1], p3[k >> 1]);
                    }
                    tmem_st_32x8(mine + 16 * c, p1);
                    tmem_st_32x8(mine + 16 * c + 8, p2);
                    tmem_st_32x8(mine + C::COL_P3 + 8 * c, p3);
                }
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(p_full(set));
                pending = true;
                last_turn = turn;
            }
            const bool ends = w.next(g.w);
            more = w.left > 0;
            if (!ends || !ok) continue;
            if (pending) {
                if (!wait_all(s_free(set), last_turn & 1)) break;
                ptx::tc_fence_after_sync();
                collect();
            }
            const long long part = part_of(blockIdx.x, (long long)o * g.w.NB + blk, set, SETS) * kTile + lane_row;
            float l0, l1;
            split(sums, l0, l1);
            f.part_ml[part] = make_float2(ref * c2, l0 + l1);   // (-inf, 0): no entries
            float *to = g.part + part * 64;
#pragma unroll
            for (int k = 0; k < 64; k += 4) *reinterpret_cast<float4 *>(to + k) = make_float4(acc[k], acc[k + 1], acc[k + 2], acc[k + 3]);
#pragma unroll
            for (int k = 0; k < 64; ++k) acc[k] = 0.f;
            sums = two(0.f, 0.f);
            ref = -CUDART_INF_F;
            pending = false;
        }
    }
    __syncwarp();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == FIRST_WARP) { ptx::tc_fence_after_sync(); ptx::tmem_dealloc(tmem, C::COLS); }
}

// A CTA per 16 rows of a block, a thread per four elements: the sums of all sets of all CTAs that had tiles of it, in order, each rescaled
// when the reference moves.
constexpr int kJoinRows32 = 16, kJoinParts32 = kTile / kJoinRows32;
template <int V, int DW>
__global__ void __launch_bounds__(256) tile_forward32_join_kernel(const __grid_constant__ Args32 f)
{
    const GradArgsOf<float> &g = f.g;
    const TileArgsOf<float> &a = g.a;
    const Shape &s = a.g.s;
    const int block = blockIdx.x / kJoinParts32, part = blockIdx.x % kJoinParts32, o = block / g.w.NB, blk = block % g.w.NB;
    const int b = o / g.w.outer, h = o % g.w.outer, row0 = blk * kTile + part * kJoinRows32;
    if (row0 >= s.M) return;
    const int pat = pattern_of(s.patterns, s.batch, s.heads, b, h);
    const int *ptr = a.g.ptr + pat * a.g.ptr_stride;
    const int col = (threadIdx.x & 15) * 4, r = threadIdx.x >> 4, row = row0 + r;
    __shared__ unsigned redo;
    if (threadIdx.x == 0) redo = 0;
    __syncthreads();
    // (of the pattern and its plan, which the kernels ahead do not write)
    int c0, c1;
    const long long n = g.holders(o, blk, c0, c1);
    const bool live = row < s.M && n > 0 && ptr[row + 1] > ptr[row];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (row < s.M) {
        float x[4] = {}, m = -CUDART_INF_F, l = 0.f;
        if (live) {
            for (int c = c0; c <= c1; ++c) {
                float2 ml[Fwd32::SETS];
                float4 v[Fwd32::SETS];
#pragma unroll
                for (int set = 0; set < Fwd32::SETS; ++set) {
                    const long long at = part_of(c, block, set, Fwd32::SETS) * kTile + part * kJoinRows32 + r;
                    ml[set] = f.part_ml[at];
                    v[set] = *reinterpret_cast<const float4 *>(g.part + at * 64 + col);
                }
#pragma unroll
                for (int set = 0; set < Fwd32::SETS; ++set) {
                    if (ml[set].x == -CUDART_INF_F && ml[set].y == 0.f) continue;   // (a NaN beside -inf: the row is taken one by one)
                    // (a reference is finite unless a product is infinite or NaN: then the row is taken one by one)
                    const float to = fmaxf(m, ml[set].x), was = ex2(m - to), w = ex2(ml[set].x - to);
                    m = to;
                    l = fmaf(ml[set].y, w, l * was);
                    x[0] = fmaf(v[set].x, w, x[0] * was); x[1] = fmaf(v[set].y, w, x[1] * was);
                    x[2] = fmaf(v[set].z, w, x[2] * was); x[3] = fmaf(v[set].w, w, x[3] * was);
                }
            }
        }
        bool bad = live && !(l >= 7.8886091e-31f && l <= 3.402823466e38f);
        const float inv = live ? 1.f / l : 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[k] *= inv;
            bad |= live && col + k < f.dc && !(fabsf(x[k]) <= 3.402823466e38f);
        }
        store4<float, V>(a.g.out1.at(b, h, row) + f.col0, col, f.dc, x);
        if (col == 0) a.g.lse[(long long)o * s.M + row] = live ? (m + log2f(l)) * kLn2 : -CUDART_INF_F;
        if (bad) atomicOr(&redo, 1u << r);
    }
    __syncthreads();
    for (unsigned left = redo >> (threadIdx.x >> 5), r = threadIdx.x >> 5; left; left >>= 8, r += 8)
        if (left & 1) take_rows_again<kForward, DW, float, V>(a.g, a.g.ptr, a.g.idx, b, h, 1, row0 + (int)r, 1u, a.g.ptr_stride, a.g.idx_stride);
}

// ---- the backward pass -------------------------------------------------------------------------------------------------------------
// Two sets of four softmax warps; eight warps that add up the second products, step by step, in registers.
template <int MODE, bool READ = false> struct Grad32 {
    static constexpr int SETS = READ && MODE == kDq ? 3 : 2, THREADS = 128 * SETS + 256 + 96, STAGES = 2, ACCS = MODE == kDkv ? 2 : 1;
    static constexpr int STAT = MODE == kDkv ? 512 : 0;
    static constexpr int X1 = 0, X2 = kPlaneTile, Y1 = 2 * kPlaneTile, Y2 = Y1 + STAGES * kPlaneHalf, ST = Y2 + STAGES * kPlaneHalf, BAR = ST + STAGES * STAT;
    static constexpr int BYTES = BAR + 512 + 1024;
    // tensor memory: sums of a step; of a set S, dP and (dK, dV) the third planes.  Planes of 16 elements k of a row: dQ: dS over S and dP; dK, dV: P over S,
    // dS over dP.
    static constexpr uint32_t COL_S = 128, SET = MODE == kDkv ? 192 : 128, COLS = 512;
    static_assert(BYTES <= 232448 && COL_S + SETS * SET <= 512, "shared or tensor memory");
    __device__ static constexpr int ds(int p, int k) { return MODE == kDq ? (p == 2 ? 64 + 16 * k : 16 * k + 8 * p) : p == 2 ? 128 + 16 * k + 8 : 64 + 16 * k + 8 * p; }
    __device__ static constexpr int pp(int p, int k) { return p == 2 ? 128 + 16 * k : 16 * k + 8 * p; }
};

template <int MODE, bool READ>
__global__ void __launch_bounds__(Grad32<MODE, READ>::THREADS, 1)
tile_grad32_kernel(const __grid_constant__ CUtensorMap tm_x1, const __grid_constant__ CUtensorMap tm_x2, const __grid_constant__ CUtensorMap tm_y1,
                   const __grid_constant__ CUtensorMap tm_y2, const __grid_constant__ Args32 f)
{
    using C = Grad32<MODE, READ>;
    constexpr int SETS = C::SETS, SUM_WARP = 4 * SETS, TMA_WARP = SUM_WARP + 8, FIRST_WARP = TMA_WARP + 1, SECOND_WARP = TMA_WARP + 2;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (ptx::smem_u32(raw) + 1023u) & ~1023u, bars = base + C::BAR;
    auto full = [&](int s) { return bars + 8u * s; };
    auto free_ = [&](int s) { return bars + 64u + 8u * s; };
    auto s_full = [&](int w) { return bars + 128u + 8u * w; };
    auto p_full = [&](int w) { return bars + 152u + 8u * w; };
    auto s_free = [&](int w) { return bars + 176u + 8u * w; };
    auto flags = [&](int s) { return bars + 320u + 4u * s; };
    const uint32_t x_full = bars + 200, x_free = bars + 208, o_full = bars + 216, o_free = bars + 224, slot = bars + 232;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const GradArgsOf<float> &g = f.g;
    const TileArgsOf<float> &a = g.a;
    const Shape &s = a.g.s;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) { ptx::mbar_init(full(i), 1); ptx::mbar_init(free_(i), 1); }
        for (int i = 0; i < SETS; ++i) { ptx::mbar_init(s_full(i), 1); ptx::mbar_init(p_full(i), 4); ptx::mbar_init(s_free(i), 1); }
        ptx::mbar_init(x_full, 1); ptx::mbar_init(x_free, 1); ptx::mbar_init(o_full, 1); ptx::mbar_init(o_free, 8);
        ptx::mbar_init(slot + 16, 1); ptx::mbar_init(slot + 24, 1);   // the last products
        ptx::fence_mbar_init();
    }
    if (warp == FIRST_WARP) { ptx::tmem_alloc(slot, C::COLS); ptx::tmem_relinquish(); }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t tmem = ptx::lds32(slot);
    const int tiles = (int)(g.first[blockIdx.x + 1] - g.first[blockIdx.x]), steps = 2 * tiles;
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !wait_for(bar, parity)) { ok = false; *a.status = B2SP_ERR_TIMEOUT; }
        return ok;
    };
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return ok = __all_sync(~0u, wait(bar, parity)); };
    if (warp == TMA_WARP) {
        Walk w;
        w.start(g.w, g.starts[blockIdx.x], tiles);
        int i = 0, blocks = 0;
        for (bool more = tiles > 0; more && ok;) {
            const int b = w.o / g.w.outer, x = w.o % g.w.outer, h = x * g.w.group + w.i, hy = MODE == kDq ? h / (s.heads / s.kv_heads) : h, blk = w.blk;
            const int r0 = (MODE == kDq ? g.tile_at[w.t] : g.tile_at[2 * w.t]) * kTile;
            if (READ) {
                const long long at = tile_number(f.rows, b * s.heads + h, MODE == kDq ? w.t : g.tile_at[2 * w.t + 1]) * kScores;
                if (ptx::elect_one()) {
                    prefetch(f.scores[0] + at, kScores * 4);
                    prefetch(f.scores[1] + at, kScores * 4);
                }
                __syncwarp();
            }
            const bool fresh = w.fresh, last = w.next(g.w);
            more = w.left > 0;
            if (!READ && fresh) {
                if (!wait_all(x_free, (blocks & 1) ^ 1)) break;
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(x_full, 2 * kPlaneTile);
                    load_planes<128>(base + C::X1, &tm_x1, x_full, 0, blk * kTile, x, b);
                    load_planes<128>(base + C::X2, &tm_x2, x_full, 0, blk * kTile, x, b);
                }
                __syncwarp();
                ++blocks;
            }
            for (int half = 0; half < 2; ++half, ++i) {
                const int st = i % C::STAGES, at = r0 + half * 64;
                if (!wait_all(free_(st), (i / C::STAGES & 1) ^ 1)) break;
                if (ptx::elect_one()) {
                    ptx::sts32(flags(st), (fresh && !half ? kStepFirst : 0) | (last && half ? kStepLast : 0));
                    constexpr bool BOTH = !READ || MODE == kDkv;   // (V serves dP alone)
                    ptx::mbar_arrive_expect_tx(full(st), (BOTH ? 2 : 1) * kPlaneHalf + C::STAT);
                    load_planes<64>(base + C::Y1 + st * kPlaneHalf, &tm_y1, full(st), f.col0 / kPlane, at, hy, b);
                    if (BOTH) load_planes<64>(base + C::Y2 + st * kPlaneHalf, &tm_y2, full(st), f.col0 / kPlane, at, hy, b);
                    if (MODE == kDkv) bulk_load(base + C::ST + st * C::STAT, a.g.stat + ((long long)b * s.heads + h) * a.g.stat_stride + at, C::STAT, full(st));
                }
                __syncwarp();
            }
        }
        // copies in flight land before the CTA ends, also where another warp gave up a wait
        if (blocks) ptx::mbar_wait(x_full, (blocks - 1) & 1);
        for (int k = max(0, i - C::STAGES); k < i; ++k) ptx::mbar_wait(full(k % C::STAGES), k / C::STAGES & 1);
    } else if (warp == FIRST_WARP) {
        if (!READ && ptx::elect_one()) {
            const int ks = (s.d + 15) >> 4;
            const uint32_t x1 = desc_columns(base + C::X1), x2 = desc_columns(base + C::X2), y1 = desc_columns(base + C::Y1), y2 = desc_columns(base + C::Y2);
            int st = 0, ph = 0, set = 0, round = 0, blocks = 0;
            for (int i = 0; i < steps; ++i) {
                if (!wait(full(st), ph)) break;
                const uint32_t fl = ptx::lds32(flags(st));
                if ((fl & kStepFirst) && !wait(x_full, blocks++ & 1)) break;
                if (round && !wait(s_free(set), (round - 1) & 1)) break;
                const uint32_t to = tmem + C::COL_S + set * C::SET;
                product_columns32<64>(to, x1, y1 + st * (kPlaneHalf >> 4), ks);
                product_columns32<64>(to + 64, x2, y2 + st * (kPlaneHalf >> 4), ks);
                ptx::mma_commit(s_full(set));
                if (fl & kStepLast) ptx::mma_commit(x_free);
                if (++st == C::STAGES) { st = 0; ph ^= 1; }
                if (++set == SETS) { set = 0; ++round; }
            }
            ptx::mma_commit(slot + 16);   // products in flight end before tensor memory is freed, also where another warp gave up a wait
            ptx::mbar_wait(slot + 16, 0);
        }
        __syncwarp();
    } else if (warp == SECOND_WARP) {
        if (ptx::elect_one()) {
            const uint32_t y1 = desc_rows<64>(base + C::Y1), y2 = desc_rows<64>(base + C::Y2);
            int st = 0, ph = 0, set = 0, round = 0;
            for (int i = 0; i < steps; ++i) {
                if (!wait(full(st), ph)) break;
                if (i && !wait(o_free, (i - 1) & 1)) break;   // the last step's sums are read
                if (!wait(p_full(set), round & 1)) break;
                ptx::tc_fence_after_sync();
                const uint32_t from = tmem + C::COL_S + set * C::SET;
                product_rows32(tmem, from, y1 + st * (kPlaneHalf >> 4), [](int p, int k) { return C::ds(p, k); });
                if (MODE == kDkv) product_rows32(tmem + 64, from, y2 + st * (kPlaneHalf >> 4), [](int p, int k) { return C::pp(p, k); });
                ptx::mma_commit(s_free(set));
                ptx::mma_commit(free_(st));
                ptx::mma_commit(o_full);
                if (++st == C::STAGES) { st = 0; ph ^= 1; }
                if (++set == SETS) { set = 0; ++round; }
            }
            ptx::mma_commit(slot + 24);   // products in flight end before tensor memory is freed, also where another warp gave up a wait
            ptx::mbar_wait(slot + 24, 0);
        }
        __syncwarp();
    } else if (warp < SUM_WARP) {
        const int set = warp >> 2, lane_row = threadIdx.x & 127;
        const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16) + C::COL_S + set * C::SET;
        const float c2 = s.scale * kLog2e;
        const uint64_t f2 = two(c2, c2);
        Walk w;
        w.start(g.w, g.starts[blockIdx.x], tiles);
        int at_set = 0, round = 0, st = 0, ph = 0;
        float2 own = make_float2(0.f, 0.f);
        for (bool more = tiles > 0; more && ok;) {
            if (MODE == kDq && w.fresh) own = a.g.stat[(long long)w.o * a.g.stat_stride + w.blk * kTile + lane_row];
            const uint4 now = __ldg((MODE == kDq ? a.plan.masks : a.plan.tmasks) + (long long)w.t * kTile + lane_row);
            const uint64_t l2 = two(own.x, own.x), d2 = two(own.y, own.y);
            for (int half = 0; half < 2; ++half) {
                const bool my_turn = at_set == set;
                const int stage = st, turn = round, at_stage = ph;
                if (++st == C::STAGES) { st = 0; ph ^= 1; }
                if (++at_set == SETS) { at_set = 0; ++round; }
                if (!my_turn) continue;
                if (READ) {   // (what the set left in tensor memory is read by then, and the statistics are there)
                    if (turn && !wait_all(s_free(set), (turn - 1) & 1)) break;
                    if (MODE == kDkv && !wait_all(full(stage), at_stage & 1)) break;
                } else if (!wait_all(s_full(set), turn & 1)) {
                    break;
                }
                ptx::tc_fence_after_sync();
                const float *sc = nullptr;
                long long dp_at = 0;
                if (READ) {
                    const int head = w.o / g.w.outer * s.heads + w.o % g.w.outer * g.w.group + w.i;
                    sc = f.scores[0] + tile_number(f.rows, head, MODE == kDq ? w.t : g.tile_at[2 * w.t + 1]) * kScores;
                    sc += MODE == kDq ? half * (64 * kTile) + lane_row : lane_row * kTile + half * 64;
                    dp_at = f.scores[1] - f.scores[0];
                }
                const uint32_t stat = base + C::ST + stage * C::STAT;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t x[16], y[16];
                    if (READ && MODE == kDq) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(sc[(16 * c + k) * kTile]);
#pragma unroll
                        for (int k = 0; k < 16; ++k) y[k] = __float_as_uint(sc[dp_at + (16 * c + k) * kTile]);
                        settle(x);   // (all in flight)
                        settle(y);
                    } else if (READ) {
#pragma unroll
                        for (int k = 0; k < 16; k += 4) {
                            const uint4 u = *reinterpret_cast<const uint4 *>(sc + 16 * c + k), v = *reinterpret_cast<const uint4 *>(sc + dp_at + 16 * c + k);
                            x[k] = u.x; x[k + 1] = u.y; x[k + 2] = u.z; x[k + 3] = u.w;
                            y[k] = v.x; y[k + 1] = v.y; y[k + 2] = v.z; y[k + 3] = v.w;
                        }
                        settle(x);   // (all in flight)
                        settle(y);
                    } else {
                        ptx::tmem_ld_32x16(from + 16 * c, x);
                        ptx::tmem_ld_32x16(from + 64 + 16 * c, y);
                        ptx::tmem_ld_wait();
                        settle(x);
                        settle(y);
                    }
                    const uint32_t m = (half ? (c & 2 ? now.w : now.z) : (c & 2 ? now.y : now.x)) >> (16 * (c & 1));
                    uint32_t p1[8], p2[8], p3[8], q1[8], q2[8], q3[8];
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        float p0, pb, e0, e1;
                        uint64_t nl = l2, nd = d2;
                        if (MODE == kDkv) {
                            float l0, d0, l1, d1;
                            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(l0), "=f"(d0), "=f"(l1), "=f"(d1) : "r"(stat + (16 * c + k) * 8));
                            nl = two(l0, l1);
                            nd = two(d0, d1);
                        }
                        split(fma2(two(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), f2, nl), p0, pb);
                        p0 = m >> k & 1 ? ex2(p0) : 0.f;
                        pb = m >> (k + 1) & 1 ? ex2(pb) : 0.f;
                        split(mul2(two(p0, pb), add2(two(__uint_as_float(y[k]), __uint_as_float(y[k + 1])), nd)), e0, e1);
                        if (MODE == kDkv) split3(p0, pb, p1[k >> 1], p2[k >> 1], p3[k >> 1]);
                        split3(e0, e1, q1[k >> 1], q2[k >> 1], q3[k >> 1]);
                    }
                    if (MODE == kDkv) {
                        tmem_st_32x8(from + C::pp(0, c), p1);
                        tmem_st_32x8(from + C::pp(1, c), p2);
                        tmem_st_32x8(from + C::pp(2, c), p3);
                    }
                    tmem_st_32x8(from + C::ds(0, c), q1);
                    tmem_st_32x8(from + C::ds(1, c), q2);
                    tmem_st_32x8(from + C::ds(2, c), q3);
                }
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(p_full(set));
            }
            w.next(g.w);
            more = w.left > 0;
        }
    } else {
        // sums: warps 0-3 the first half of the columns (dQ) or dK, warps 4-7 the second half or dV
        constexpr int N = MODE == kDkv ? 64 : 32;
        const int which = (warp - SUM_WARP) >> 2, lane_row = threadIdx.x & 127, acc_of = MODE == kDkv ? which : 0, col0 = MODE == kDkv ? 0 : which * 32;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16) + which * N;
        float acc[N];
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] = 0.f;
        Walk w;
        w.start(g.w, g.starts[blockIdx.x], tiles);
        int i = 0, first_i = w.i, first_t = w.t;
        unsigned some = 0;
        for (bool more = tiles > 0; more && ok;) {
            const int blk = w.blk, o = w.o;
            if (w.fresh) {
                some = 0;
                first_i = w.i;
                first_t = w.t;
            }
            const uint4 now = __ldg((MODE == kDq ? a.plan.masks : a.plan.tmasks) + (long long)w.t * kTile + lane_row);
            some |= now.x | now.y | now.z | now.w;
            for (int half = 0; half < 2; ++half, ++i) {
                if (!wait_all(o_full, i & 1)) break;
                ptx::tc_fence_after_sync();
#pragma unroll
                for (int c = 0; c < N; c += 16) {
                    uint32_t x[16];
                    ptx::tmem_ld_32x16(mine + c, x);
                    ptx::tmem_ld_wait();
                    settle(x);
#pragma unroll
                    for (int k = 0; k < 16; ++k) acc[c + k] += __uint_as_float(x[k]);
                }
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(o_free);
            }
            const int last_i = w.i;
            const bool ended = w.t + 1 == w.t1, ends = w.next(g.w);
            more = w.left > 0;
            if (!ends || !ok) continue;
            const int rows = MODE == kDq ? s.M : s.K, row = blk * kTile + lane_row, b = o / g.w.outer, h = o % g.w.outer;
            bool begun = true, whole = true;
            for (int k = 0; k <= first_i; ++k) {
                const int p = g.w.pattern(o, k), t0 = g.w.at(p, blk);
                if (k < first_i ? g.w.at(p, blk + 1) > t0 : first_t > t0) begun = false;
            }
            whole = begun && ended;
            for (int k = last_i + 1; k < g.w.group && whole; ++k) {
                const int p = g.w.pattern(o, k);
                if (g.w.at(p, blk + 1) > g.w.at(p, blk)) whole = false;
            }
            bool bad = false;
            if (whole) {
                if (row < rows) {
                    float *to = (acc_of ? a.g.out2 : a.g.out1).at(b, h, row) + f.col0;
                    const float by = acc_of ? 1.f : s.scale;
#pragma unroll
                    for (int k = 0; k < N; k += 4) {
                        float x[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[e] = some ? acc[k + e] * by : 0.f;
                            bad |= col0 + k + e < f.dc && !(fabsf(x[e]) <= 3.402823466e38f);
                        }
                        if (f.wide) store4<float, 4>(to, col0 + k, f.dc, x);
                        else store4<float, 1>(to, col0 + k, f.dc, x);
                    }
                }
            } else {
                float *to = g.part + ((((long long)blockIdx.x * 2 + begun) * C::ACCS + acc_of) * kTile + lane_row) * 64 + col0;
#pragma unroll
                for (int k = 0; k < N; k += 4) *reinterpret_cast<float4 *>(to + k) = make_float4(acc[k], acc[k + 1], acc[k + 2], acc[k + 3]);
            }
            if (bad) g.bad[(long long)o * g.w.NB + blk] = 1;
#pragma unroll
            for (int k = 0; k < N; ++k) acc[k] = 0.f;
        }
    }
    __syncwarp();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == FIRST_WARP) { ptx::tc_fence_after_sync(); ptx::tmem_dealloc(tmem, C::COLS); }
}

}  // namespace attn
}  // namespace b2sp
