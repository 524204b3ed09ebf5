// Attention over the tiles of a plan on the tensor cores (tcgen05, tensor memory, TMA): bfloat16, head widths up to 128.
//
// At the densities that masks have (10% to 30% scattered, or dense inside a window) a 128 x 128 tile of the pattern is cheaper multiplied
// whole than entry by entry: what is not stored is masked by the tile's 128 x 128 bits, which the plan holds ready.  Tiles without an entry are never
// visited.
//   forward  a CTA per 128 rows, 64 keys a step, two CTAs per SM: S = Q K^T into one of two places in tensor memory; each thread of four softmax
//            warps takes a row, masks, exponentiates and writes the weights over S as bfloat16; O += P V accumulates in tensor memory.
//   backward dQ, then dK with dV: see there.  Two passes over the tiles (seven products instead of five, the weights twice) need neither
//            atomics nor a slab of fp32 gradients, so results are the same bits every time.
//
// What bounds the forward pass at width 64: the exponentials (16 a clock on an SM: 1024 clocks a tile of 128 x 128) and what stands around them, 64 us for
// 8 x 4096 x 4096 at 20% (their unit is busy 54% to 68% of the time); at width 128 the tensor core (two products of 512 clocks a tile) is as
// long: 83 us for 16 heads over 4 of 8192 under a window of 1024, 820 Tflop/s of the stored entries.
//
// The reference of the exponentials (the "maximum") is taken over all 128 products of a row's tile, masked or not, which spares the mask in
// that sweep; it moves only when it grows by more than 8 (to base 2), so O is rarely rescaled.  A row that loses its weights to
// a larger masked product (their sum below 2^-100), or meets a NaN or an infinity -- a masked weight of 0 times a row of V that holds one, which
// no entry names, is NaN -- is computed again entry by entry, by the row kernels' code.  Results are thus those of the stored entries alone, but
// the reference rounds the exponents' arguments: 2^-18 of a weight at most, with the weight's own rounding to bfloat16 at 2^-8.  (A reference of the
// stored products alone, found where all products exceed the last one: 7.8 -> 8.6 us for four heads of 256 x 256, 63.8 -> 64.1 for 8 x 4096.)
#pragma once
#include <cuda.h>

#include "attention_tiles.h"
#include "ptx_sm100.cuh"

namespace b2sp {
namespace attn {

struct Op {              // a tensor map's coordinates of (b, h): 0 where the operand is shared
    int hm, bm;
};

template <typename T> struct TileArgsOf {
    RowArgs<T> g;        // operands, pattern and outputs for rows that are taken one by one
    Plan plan;
    Op q, k, v, dout;
    const int *col_ptr, *row_idx;        // transposed pattern
    int *status;
};
using TileArgs = TileArgsOf<Bf16>;

// Bounded wait that asks for a complete phase with a test first (36 cycles; the try_wait of ptx::mbar_wait answers in 92).
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0 || ptx::mbar_wait(bar, parity);
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void *tmap, uint32_t bar, int c0, int c1, int c2, int c3)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar) : "memory");
}
// bf16 x bf16 -> fp32, M = 128 rows, N columns; B along K (rows of K elements) or along N.
__host__ __device__ constexpr uint32_t idesc_bf16(int N, bool b_along_n)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_along_n ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | (8u << 24);
}
// Descriptors of shared-memory operands come as their lower halves (the upper one is the same for all): steps along an operand are
// 32-bit additions.
constexpr uint32_t kDescHigh = (1024u >> 4) | 1u << 14 | ptx::kLayoutSw128 << 29;   // eight rows 1024 bytes apart, version 1, 128-byte swizzle
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tmov.b64 y, {%2, %5};\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHigh) : "memory");
}
__device__ __forceinline__ void tmem_st_32x8(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// After tmem_ld_wait(): nothing that uses the loaded registers moves in front of the wait.
__device__ __forceinline__ void settle(uint32_t (&x)[32])
{
    asm volatile("" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]), "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15]), "+r"(x[16]), "+r"(x[17]), "+r"(x[18]), "+r"(x[19]), "+r"(x[20]), "+r"(x[21]), "+r"(x[22]), "+r"(x[23]), "+r"(x[24]), "+r"(x[25]), "+r"(x[26]), "+r"(x[27]), "+r"(x[28]), "+r"(x[29]), "+r"(x[30]), "+r"(x[31]));
}

__device__ __forceinline__ void settle(uint32_t (&x)[16])
{
    asm volatile("" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]), "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15]));
}

// Operand tiles in shared memory: blocks of 64 columns, each ROWS rows of 128 bytes, 128-byte swizzle.  The same bytes are an operand whose
// contraction runs along the columns (steps of 16: 32 bytes) or along the rows (steps of 16: 2 KB; blocks of 64 columns ROWS * 128 bytes apart).
__device__ __forceinline__ uint32_t desc_columns(uint32_t base) { return base >> 4 | 1u << 16; }
template <int ROWS> __device__ __forceinline__ uint32_t desc_rows(uint32_t base) { return base >> 4 | (ROWS * 128u >> 4) << 16; }
template <int ROWS> __host__ __device__ constexpr uint32_t column_step(int k) { return ((k >> 2) * (ROWS * 128) + (k & 3) * 32) >> 4; }
__host__ __device__ constexpr uint32_t row_step(int k) { return k * 2048 >> 4; }
// D = A B^T over DP columns (those behind `ks` steps of 16 are zeros), A 128 rows, B N rows.
template <int DP, int N> __device__ __forceinline__ void product_columns(uint32_t d, uint32_t a, uint32_t b, int ks)
{
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
        if (k < ks) mma_ss(d, a + column_step<128>(k), b + column_step<N>(k), idesc_bf16(N, false), k > 0);
}
// D (+)= A B, A 128 x ROWS in tensor memory (32 elements of a row in 16 columns; the next 32 follow SKIP columns on), B ROWS x DP.
template <int DP, int ROWS, int SKIP = 16> __device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, uint32_t b, bool onto)
{
#pragma unroll
    for (int k = 0; k < ROWS / 16; ++k) mma_ts(d, a + (k >> 1) * SKIP + (k & 1) * 8, b + row_step(k), idesc_bf16(DP, true), k > 0 || onto);
}
template <int DP, int ROWS> __device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *tm, uint32_t bar, int row, int h, int b)
{
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) tma_load_4d(dst + c * ROWS * 128, tm, bar, c * 64, row, h, b);
}

// 32 accumulator columns of a thread's row times f, as bfloat16.  Returns whether all are finite.
__device__ __forceinline__ bool store32(Bf16 *row, int c0, int d, const uint32_t (&x)[32], float f)
{
    bool fine = true;
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            y[k] = __uint_as_float(x[i + k]) * f;
            fine &= fabsf(y[k]) <= 3.402823466e38f;
        }
        if (c0 + i < d)
            *reinterpret_cast<uint4 *>(row + c0 + i) = make_uint4(bf16x2(y[0], y[1]), bf16x2(y[2], y[3]), bf16x2(y[4], y[5]), bf16x2(y[6], y[7]));
    }
    return fine;
}

// Rows of the 32 that a warp owns whose lane says `bad`, entry by entry (rows of the pattern; kGradKV: columns, over the query heads
// [h0, h0 + heads) that share them).
template <int MODE, int DW, typename T, int V>
__device__ __noinline__ void rows_one_by_one(const RowArgs<T> &g, const int *ptr, const int *idx, int b, int h0, int heads, int row0, unsigned bad,
                                             long long ptr_stride, long long idx_stride)
{
    for (; bad; bad &= bad - 1) {
        const int row = row0 + __ffs(bad) - 1;
        RowWork<MODE, T, V, DW> w, all;
        for (int i = 0; i < heads; ++i) {
            const int pat = pattern_of(g.s.patterns, g.s.batch, g.s.heads, b, h0 + i);
            const int *p = ptr + pat * ptr_stride;
            w.run(g, b, h0 + i, row, idx + pat * idx_stride, p[row], p[row + 1]);
            if (MODE == kGradKV && i) {
#pragma unroll
                for (int u = 0; u < w.AU; ++u)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        all.acc1[u][k] += w.acc1[u][k];
                        if constexpr (MODE == kGradKV) all.acc2[u][k] += w.acc2[u][k];
                    }
            } else {
                all = w;
            }
        }
        all.finish(g, b, h0, row);
    }
}
// The same for a kernel that stores the outputs in groups of V.  Those rows are read as they lie: fp32 inputs may have any alignment beside
// aligned outputs.
template <int MODE, int DW, typename T, int V>
__device__ __forceinline__ void take_rows_again(const RowArgs<T> &g, const int *ptr, const int *idx, int b, int h0, int heads, int row0, unsigned bad,
                                                long long ptr_stride, long long idx_stride)
{
    if (V == 4 && (sizeof(T) == 2 || g.fours_in)) rows_one_by_one<MODE, DW, T, 4>(g, ptr, idx, b, h0, heads, row0, bad, ptr_stride, idx_stride);
    else rows_one_by_one<MODE, DW, T, sizeof(T) == 2 ? 4 : 1>(g, ptr, idx, b, h0, heads, row0, bad, ptr_stride, idx_stride);
}

constexpr int kTileThreads = 192;   // four softmax warps, a TMA warp, an MMA warp

// ---- forward ---------------------------------------------------------------------------------------------------------------------
// A CTA per (problem, row block), two per SM; 64 keys a step.  S has two buffers in tensor memory, so that the products of the next step are
// there when the softmax warps come to it; the weights (bfloat16) lie over the S that they come from.
// Not kept: eight softmax warps with 32 keys each, which tell each other their largest products (eight problems of 4096 x 4096 at 20%, d = 64:
// 63 -> 70 us), and the next step's products fetched and compared among the exponentials of this one (64 -> 70 us, 168 registers).
template <int DP> struct FwdCfg {
    static constexpr int KSTAGES = DP == 64 ? 4 : 3, VSTAGES = DP == 64 ? 4 : 2;   // (K is read two steps ahead of V)
    static constexpr int TILE = 128 * DP * 2, HALF = 64 * DP * 2;
    // (without room to align in: two CTAs at width 128 take all of an SM's shared memory, which begins on a multiple of 1024 bytes)
    static constexpr int Q = 0, K = TILE, V = K + KSTAGES * HALF, BAR = V + VSTAGES * HALF, BYTES = BAR + 256;
    static constexpr uint32_t COL_S = 0, COL_O = 128, COLS = 256;
};

// Few blocks with many tiles each are cut into parts (SPLIT): each leaves its sums and its reference, which the kernel below joins.  128 queries
// of 8 heads over 8192 keys, width 128, 50%: 86 us whole, 17 us in parts; four heads of 4096, causal, width 64 (128 blocks): 48 and 36 us.
struct FwdParts {
    int splits;
    float *part;        // [block][splits][128][DP]
    float2 *part_ml;    // [block][splits][128]: reference (to base 2), sum; (-inf, 0): no entries
};
template <int DP, bool SPLIT>
__global__ void __launch_bounds__(kTileThreads, 2)
tile_forward_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ TileArgs a, const FwdParts f)
{
    using C = FwdCfg<DP>;
    extern __shared__ __align__(1024) uint8_t aligned_raw[];
    const uint32_t base = ptx::smem_u32(aligned_raw), bars = base + C::BAR;
    auto k_full = [&](int s) { return bars + 8u * s; };
    auto k_free = [&](int s) { return bars + 32u + 8u * s; };
    auto v_full = [&](int s) { return bars + 64u + 8u * s; };
    auto v_free = [&](int s) { return bars + 96u + 8u * s; };
    auto s_full = [&](int b) { return bars + 128u + 8u * b; };
    auto p_full = [&](int b) { return bars + 144u + 8u * b; };   // (one per buffer: a fast warp may be a step ahead of a slow one)
    const uint32_t q_full = bars + 160, o_full = bars + 168, slot = bars + 176, done = bars + 192;   // o_full: after every step's second product; done: after the last
    const int warp = threadIdx.x >> 5;
    const Shape &s = a.g.s;
    const int problems = s.batch * s.heads, RB = a.plan.RB;
    const int part = SPLIT ? blockIdx.x % f.splits : 0, block = SPLIT ? blockIdx.x / f.splits : blockIdx.x;
    const int prob = block % problems, rb = RB - 1 - block / problems;   // (a causal mask's longest rows first)
    const int b = prob / s.heads, h = prob % s.heads, hkv = h / (s.heads / s.kv_heads);
    const int pat = pattern_of(s.patterns, s.batch, s.heads, b, h);
    int t0 = a.plan.rb_ptr[pat * RB + rb], steps = 2 * (a.plan.rb_ptr[pat * RB + rb + 1] - t0);
    const long long rows_at = ((long long)block * f.splits + part) * kTile + threadIdx.x;   // of a softmax thread's sums
    if (SPLIT) {
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        const int per = (steps / 2 + f.splits - 1) / f.splits, ahead = min(part * per, steps / 2);
        t0 += ahead;
        steps = 2 * min(per, steps / 2 - ahead);
    }
    const int row = rb * kTile + threadIdx.x;   // of a softmax thread
    float *lse = a.g.lse + (long long)prob * s.M;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
    if (SPLIT && steps == 0) {
        if (threadIdx.x < 128) f.part_ml[rows_at] = make_float2(-CUDART_INF_F, 0.f);
        return;
    }
    if (steps == 0) {
        if (threadIdx.x < 128 && row < s.M) {
            Bf16 *o = a.g.out1.at(b, h, row);
            for (int c = 0; c < s.d; c += 8) *reinterpret_cast<uint4 *>(o + c) = make_uint4(0, 0, 0, 0);
            lse[row] = -CUDART_INF_F;
        }
        return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::KSTAGES; ++i) { ptx::mbar_init(k_full(i), 1); ptx::mbar_init(k_free(i), 1); }
        for (int i = 0; i < C::VSTAGES; ++i) { ptx::mbar_init(v_full(i), 1); ptx::mbar_init(v_free(i), 1); }
        ptx::mbar_init(s_full(0), 1); ptx::mbar_init(s_full(1), 1);
        ptx::mbar_init(q_full, 1); ptx::mbar_init(p_full(0), 4); ptx::mbar_init(p_full(1), 4); ptx::mbar_init(o_full, 1);
        ptx::mbar_init(done, 1);
        ptx::mbar_init(slot + 8, 1);   // the last products
        ptx::fence_mbar_init();
    }
    if (warp == 5) { ptx::tmem_alloc(slot, C::COLS); ptx::tmem_relinquish(); }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = ptx::lds32(slot);
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !wait_for(bar, parity)) { ok = false; *a.status = B2SP_ERR_TIMEOUT; }
        return ok;
    };
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return ok = __all_sync(~0u, wait(bar, parity)); };   // of a softmax warp
    if (warp == 4) {
        if (ptx::elect_one()) {
            ptx::mbar_arrive_expect_tx(q_full, C::TILE);
            load_tile<DP, 128>(base + C::Q, &tm_q, q_full, rb * kTile, h * a.q.hm, b * a.q.bm);
            // K runs ahead of V by the stages that it has more
            constexpr int AHEAD = C::KSTAGES - C::VSTAGES;
            int ik = 0, iv = 0;
            auto key = [&](int i) { return a.plan.tile_cb[t0 + (i >> 1)] * kTile + (i & 1) * 64; };
            int at_k = key(0), at_v = at_k;
            while (iv < steps) {
                if (ik < steps && ik <= iv + AHEAD) {
                    const int st = ik % C::KSTAGES;
                    if (!wait(k_free(st), (ik / C::KSTAGES & 1) ^ 1)) break;
                    ptx::mbar_arrive_expect_tx(k_full(st), C::HALF);
                    load_tile<DP, 64>(base + C::K + st * C::HALF, &tm_k, k_full(st), at_k, hkv * a.k.hm, b * a.k.bm);
                    if (++ik < steps) at_k = key(ik);
                } else {
                    const int st = iv % C::VSTAGES;
                    if (!wait(v_free(st), (iv / C::VSTAGES & 1) ^ 1)) break;
                    ptx::mbar_arrive_expect_tx(v_full(st), C::HALF);
                    load_tile<DP, 64>(base + C::V + st * C::HALF, &tm_v, v_full(st), at_v, hkv * a.v.hm, b * a.v.bm);
                    if (++iv < steps) at_v = key(iv);
                }
            }
            // copies in flight land before the CTA ends, also where another warp gave up a wait
            ptx::mbar_wait(q_full, 0);
            for (int k = max(0, ik - C::KSTAGES); k < ik; ++k) ptx::mbar_wait(k_full(k % C::KSTAGES), k / C::KSTAGES & 1);
            for (int k = max(0, iv - C::VSTAGES); k < iv; ++k) ptx::mbar_wait(v_full(k % C::VSTAGES), k / C::VSTAGES & 1);
        }
        __syncwarp();
    } else if (warp == 5) {
        if (ptx::elect_one()) {
            const int ks = (s.d + 15) >> 4;
            const uint32_t q = desc_columns(base + C::Q), k0 = desc_columns(base + C::K), v0 = desc_rows<64>(base + C::V);
            auto first = [&](int i) {
                const int st = i % C::KSTAGES;
                product_columns<DP, 64>(tmem + C::COL_S + (i & 1) * 64, q, k0 + st * (C::HALF >> 4), ks);
                ptx::mma_commit(k_free(st));
                ptx::mma_commit(s_full(i & 1));
            };
            wait(q_full, 0);
            for (int i = 0; i < 2 && i < steps; ++i)
                if (wait(k_full(i % C::KSTAGES), 0)) first(i);
            for (int i = 0; i < steps && ok; ++i) {
                const int st = i % C::VSTAGES, n = i + 2;
                // everything that the next products wait for, so that both are issued as soon as the weights are there
                if (!wait(v_full(st), i / C::VSTAGES & 1)) break;
                if (n < steps && !wait(k_full(n % C::KSTAGES), n / C::KSTAGES & 1)) break;
                if (!wait(p_full(i & 1), i >> 1 & 1)) break;
                ptx::tc_fence_after_sync();
                product_rows<DP, 64>(tmem + C::COL_O, tmem + C::COL_S + (i & 1) * 64, v0 + st * (C::HALF >> 4), i > 0);
                ptx::mma_commit(v_free(st));
                ptx::mma_commit(o_full);
                if (i + 1 == steps) ptx::mma_commit(done);   // (a warp may come too late to tell the last phase of o_full from the one before)
                if (n < steps) first(n);   // (over the weights just taken: the tensor core takes one thread's products in order)
            }
            ptx::mma_commit(slot + 8);   // products in flight end before tensor memory is freed, also where another warp gave up a wait
            ptx::mbar_wait(slot + 8, 0);
        }
        __syncwarp();
    } else {
        const float c2 = s.scale * kLog2e;
        const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16);
        const uint4 *mask = a.plan.masks + (long long)t0 * kTile + threadIdx.x;
        uint4 bits = __ldg(mask), now = bits;
        float ref = 0.f;                       // reference of the exponentials, of the products before scaling
        uint64_t sums = two(0.f, 0.f);
        const uint64_t f2 = two(c2, c2);
        unsigned some = 0;
        for (int i = 0; i < steps; ++i) {
            if (!(i & 1)) {
                now = bits;
                some |= now.x | now.y | now.z | now.w;
                if (i + 2 < steps) bits = __ldg(mask + (long long)((i >> 1) + 1) * kTile);
            }
            const uint32_t from = mine + C::COL_S + (i & 1) * 64;
            if (!wait_all(s_full(i & 1), i >> 1 & 1)) break;
            ptx::tc_fence_after_sync();
            uint32_t x[2][32];
            ptx::tmem_ld_32x32(from, x[0]);
            ptx::tmem_ld_32x32(from + 32, x[1]);
            ptx::tmem_ld_wait();
            settle(x[0]);
            settle(x[1]);
            float tops[4];   // (four chains: one is 32 dependent steps)
#pragma unroll
            for (int k = 0; k < 4; ++k) tops[k] = fmaxf(__uint_as_float(x[0][k]), __uint_as_float(x[1][k]));
#pragma unroll
            for (int k = 4; k < 32; ++k) tops[k & 3] = fmaxf(tops[k & 3], fmaxf(__uint_as_float(x[0][k]), __uint_as_float(x[1][k])));
            const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
            if (__any_sync(~0u, i == 0 || (top - ref) * c2 > 8.f)) {
                const float to = top == -CUDART_INF_F ? ref : i == 0 ? top : fmaxf(top, ref), fall = i == 0 ? 0.f : ex2((ref - to) * c2);
                ref = to;
                const uint64_t fall2 = two(fall, fall);
                sums = mul2(sums, fall2);
                if (i) {
                    if (!wait_all(o_full, (i - 1) & 1)) break;   // the last step's second product
                    ptx::tc_fence_after_sync();
#pragma unroll 1
                    for (int c = 0; c < DP; c += 16) {
                        uint32_t y[16];
                        ptx::tmem_ld_32x16(mine + C::COL_O + c, y);
                        ptx::tmem_ld_wait();
                        settle(y);
#pragma unroll
                        for (int k = 0; k < 16; k += 2) {
                            float y0, y1;
                            split(mul2(two(__uint_as_float(y[k]), __uint_as_float(y[k + 1])), fall2), y0, y1);
                            y[k] = __float_as_uint(y0);
                            y[k + 1] = __float_as_uint(y1);
                        }
                        ptx::tmem_st_32x16(mine + C::COL_O + c, y);
                    }
                }
            }
            const uint64_t r2 = two(-ref * c2, -ref * c2);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const uint32_t m = (i & 1) ? (c ? now.w : now.z) : (c ? now.y : now.x);
                // all exponentials first, masked ones too (the reference bounds them): a chain per element that waits for its exponential
                // is what the loop otherwise becomes
                uint32_t p[16];
                float e[32];
#pragma unroll
                for (int k = 0; k < 32; k += 2) {
                    split(fma2(two(__uint_as_float(x[c][k]), __uint_as_float(x[c][k + 1])), f2, r2), e[k], e[k + 1]);
                    e[k] = ex2(e[k]);
                    e[k + 1] = ex2(e[k + 1]);
                }
#pragma unroll
                for (int k = 0; k < 32; k += 2) {
                    const float y0 = m >> k & 1 ? e[k] : 0.f, y1 = m >> (k + 1) & 1 ? e[k + 1] : 0.f;
                    sums = add2(sums, two(y0, y1));
                    p[k >> 1] = bf16x2(y0, y1);
                }
                ptx::tmem_st_32x16(from + 16 * c, p);
            }
            ptx::tmem_st_wait();
            ptx::tc_fence_before_sync();
            __syncwarp();
            if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(p_full(i & 1));   // (one arrival per warp: 32 on one word take turns)
        }
        wait_all(done, 0);
        ptx::tc_fence_after_sync();
        float l, l1;
        split(sums, l, l1);
        l += l1;
        if (SPLIT) {
            f.part_ml[rows_at] = some ? make_float2(ref * c2, l) : make_float2(-CUDART_INF_F, 0.f);
            float *to = f.part + rows_at * DP;
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
                uint32_t x[32];
                ptx::tmem_ld_32x32(mine + C::COL_O + c, x);
                ptx::tmem_ld_wait();
                settle(x);
#pragma unroll
                for (int k = 0; k < 32; k += 4) *reinterpret_cast<uint4 *>(to + c + k) = make_uint4(x[k], x[k + 1], x[k + 2], x[k + 3]);
            }
        }
        const bool in = !SPLIT && row < s.M, live = in && some;
        bool bad = live && !(l >= 7.8886091e-31f && l <= 3.402823466e38f);
        const float inv = live ? 1.f / l : 0.f;
        Bf16 *o = a.g.out1.at(b, h, in ? row : 0);
#pragma unroll 1
        for (int c = 0; c < (SPLIT ? 0 : DP); c += 32) {
            uint32_t x[32];
            ptx::tmem_ld_32x32(mine + C::COL_O + c, x);
            ptx::tmem_ld_wait();
            settle(x);
            if (live) bad |= !store32(o, c, s.d, x, inv);
            else if (in)
                for (int k = c; k < min(c + 32, s.d); k += 8) *reinterpret_cast<uint4 *>(o + k) = make_uint4(0, 0, 0, 0);
        }
        if (in) lse[row] = live ? fmaf(ref, c2, log2f(l)) * kLn2 : -CUDART_INF_F;
        const unsigned redo = __ballot_sync(~0u, bad);
        __syncwarp();   // (other lanes write these rows again)
        if (redo && ok) take_rows_again<kForward, DP, Bf16, 4>(a.g, a.g.ptr, a.g.idx, b, h, 1, rb * kTile + warp * 32, redo, a.g.ptr_stride, a.g.idx_stride);
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 5) { ptx::tc_fence_after_sync(); ptx::tmem_dealloc(tmem, C::COLS); }
}

// A thread per four elements of a row; parts in order, each rescaled when the reference moves.
template <int DP> __global__ void __launch_bounds__(256) tile_forward_join_kernel(const __grid_constant__ TileArgs a, const FwdParts f)
{
    constexpr int LANES = DP / 4, ROWS = 256 / LANES, PARTS = kTile / ROWS;
    const Shape &s = a.g.s;
    const int problems = s.batch * s.heads, block = blockIdx.x / PARTS, prob = block % problems, rb = a.plan.RB - 1 - block / problems;
    const int b = prob / s.heads, h = prob % s.heads, r = blockIdx.x % PARTS * ROWS + threadIdx.x / LANES, row = rb * kTile + r, col = threadIdx.x % LANES * 4;
    const int *ptr = a.g.ptr + pattern_of(s.patterns, s.batch, s.heads, b, h) * a.g.ptr_stride;
    __shared__ unsigned redo;
    if (threadIdx.x == 0) redo = 0;
    __syncthreads();
    const bool live = row < s.M && ptr[row + 1] > ptr[row];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float x[4] = {}, m = -CUDART_INF_F, l = 0.f;
    if (live) {
        const long long first = (long long)block * f.splits * kTile + r;
#pragma unroll 4
        for (int p = 0; p < f.splits; ++p) {
            const float2 ml = f.part_ml[first + p * kTile];
            if (ml.x == -CUDART_INF_F) continue;
            const float4 v = *reinterpret_cast<const float4 *>(f.part + (first + p * kTile) * DP + col);
            const float to = fmaxf(m, ml.x), was = ex2(m - to), w = ex2(ml.x - to);
            m = to;
            l = fmaf(ml.y, w, l * was);
            x[0] = fmaf(v.x, w, x[0] * was); x[1] = fmaf(v.y, w, x[1] * was);
            x[2] = fmaf(v.z, w, x[2] * was); x[3] = fmaf(v.w, w, x[3] * was);
        }
    }
    if (row < s.M) {
        bool bad = live && !(l >= 7.8886091e-31f && l <= 3.402823466e38f);
        const float inv = live ? 1.f / l : 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[k] *= inv;
            bad |= live && col + k < s.d && !(fabsf(x[k]) <= 3.402823466e38f);
        }
        store4<Bf16, 4>(a.g.out1.at(b, h, row), col, s.d, x);
        if (col == 0) a.g.lse[(long long)prob * s.M + row] = live ? (m + log2f(l)) * kLn2 : -CUDART_INF_F;
        if (bad) atomicOr(&redo, 1u << threadIdx.x / LANES);
    }
    __syncthreads();
    const int row0 = rb * kTile + blockIdx.x % PARTS * ROWS;
    for (unsigned left = redo >> (threadIdx.x >> 5), k = threadIdx.x >> 5; left; left >>= 8, k += 8)
        if (left & 1) take_rows_again<kForward, DP, Bf16, 4>(a.g, a.g.ptr, a.g.idx, b, h, 1, row0 + (int)k, 1u, a.g.ptr_stride, a.g.idx_stride);
}

// ---- the backward pass: dQ, and dK with dV -----------------------------------------------------------------------------------------
// Both walk tiles with two operands of a block of 128 rows resident (X) and two streaming by, 64 rows a step (Y):
//   dQ       X1 = Q, X2 = dO; Y1 = K, Y2 = V;   S = X1 Y1^T, dP = X2 Y2^T;              dQ += dS Y1
//   dK, dV   X1 = K, X2 = V;  Y1 = Q, Y2 = dO;  S^T = X1 Y1^T, dP^T = X2 Y2^T (rows: keys); dK += dS^T Y1, dV += P^T Y2
// Sets of eight softmax warps (two per quarter of the rows, 32 columns each) take alternate steps, each set with S and dP of its own in tensor
// memory, so that the tensor core works on the next steps while one is exponentiated; the second products' A operand (bfloat16) lies
// over what its warp has read of S and dP.
//
// Work is dealt by tiles: the tiles of all blocks in one order (problem, block, query head of the group, tile), to each CTA as many as cost `share` with what
// the blocks cost that begin there (loading X, the sums' way out), so
// that blocks of any lengths -- the keys that every query sees -- keep all SMs busy.  A block that lies in one share is finished there; of others each CTA leaves a
// part in fp32: in slot 0 if the block began in an earlier share, in slot 1 if it begins in this one; tile_grad_join_kernel adds them up in order.
enum { kDq = 0, kDkv = 1 };

// Tiles of the pattern by block (rb_ptr or cb_ptr) and who uses them.  An outer problem is a (sequence, query head) for dQ, a (sequence,
// key head) with its group of query heads for dK and dV.
struct Tiles {
    const int *ptr;
    int NB, outer, group, patterns, batch, heads, outers;
    int per;   // what a block costs beside its tiles, in tiles
    __device__ __forceinline__ int pattern(int o, int i) const { return pattern_of(patterns, batch, heads, o / outer, o % outer * group + i); }
    __device__ __forceinline__ int at(int pat, int blk) const { return ptr[(long long)pat * NB + blk]; }
    // tiles ahead of outer problem o
    __device__ __forceinline__ long long base(int o) const
    {
        const int b = o / outer, x = o % outer;
        if (patterns == 1) return (long long)o * group * at(1, 0);
        if (patterns == batch) {
            const long long t = at(b, 0);
            return group * (outer * t + (x ? x * (at(b + 1, 0) - t) : 0));
        }
        return at(b * heads + x * group, 0);
    }
    // tiles of outer problem o ahead of its block blk
    __device__ __forceinline__ long long ahead(int o, int blk) const
    {
        if (patterns == 1 || patterns == batch) {
            const int p = pattern(o, 0);
            return (long long)group * (at(p, blk) - at(p, 0));
        }
        long long n = 0;
        for (int i = 0; i < group; ++i) {
            const int p = pattern(o, i);
            n += at(p, blk) - at(p, 0);
        }
        return n;
    }
};

// The number of the first tile of the share that begins at cost `pos`: blocks cost `per` ahead of their tiles.
__device__ __forceinline__ long long share_tile(const Tiles &w, long long pos)
{
    const long long each = (long long)w.per * w.NB;
    int lo = 0, hi = w.outers;
    while (hi - lo > 1) {
        const int m = lo + ((hi - lo) >> 1);
        if (w.base(m) + each * m <= pos) lo = m; else hi = m;
    }
    const int o = lo;
    const long long before = w.base(o);
    pos -= before + each * o;
    lo = 0, hi = w.NB;
    while (hi - lo > 1) {
        const int m = lo + ((hi - lo) >> 1);
        if (w.ahead(o, m) + (long long)w.per * m <= pos) lo = m; else hi = m;
    }
    const long long ahead = w.ahead(o, lo);
    return before + ahead + max(0ll, pos - ahead - (long long)w.per * (lo + 1));
}
// Where tile number `pos` lies: (outer problem, block, query head of the group, tile).
__device__ __forceinline__ int4 share_start(const Tiles &w, long long pos)
{
    int lo = 0, hi = w.outers;
    while (hi - lo > 1) {
        const int m = lo + ((hi - lo) >> 1);
        if (w.base(m) <= pos) lo = m; else hi = m;
    }
    // (of problems without tiles, which share a base, the last one: it is the one with tiles behind `pos`)
    const int o = lo;
    pos -= w.base(o);
    lo = 0, hi = w.NB;
    while (hi - lo > 1) {
        const int m = lo + ((hi - lo) >> 1);
        if (w.ahead(o, m) <= pos) lo = m; else hi = m;
    }
    pos -= w.ahead(o, lo);
    int i = 0, t = 0;
    for (; i < w.group; ++i) {
        const int p = w.pattern(o, i), t0 = w.at(p, lo), n = w.at(p, lo + 1) - t0;
        t = t0 + (int)pos;
        if (pos < n) break;
        pos -= n;
    }
    return make_int4(o, lo, i, t);
}

// A warp's walk over its CTA's tiles; all lanes hold the same state.
struct Walk {
    int o, blk, i, t, t1, left;   // the tile at hand: query head i of the group, tile t of [.., t1); tiles left, this one included
    bool fresh;                   // it is the first of its block here
    __device__ __forceinline__ void start(const Tiles &w, int4 at, int n)
    {
        o = at.x; blk = at.y; i = at.z; t = at.w; left = n; fresh = true;
        t1 = w.at(w.pattern(o, i), blk + 1);
    }
    // Whether the next tile (if there is one) is of another block; moves on to it.
    __device__ __forceinline__ bool next(const Tiles &w)
    {
        fresh = false;
        if (--left == 0) return true;
        if (++t < t1) return false;
        while (++i < w.group) {
            const int p = w.pattern(o, i);
            t = w.at(p, blk);
            t1 = w.at(p, blk + 1);
            if (t < t1) return false;
        }
        // the next block with tiles: 32 blocks at a time
        const int lane = threadIdx.x & 31;
        fresh = true;
        ++blk;
        for (;;) {
            if (blk >= w.NB) { blk = 0; ++o; }
            if (o >= w.outers) {   // (fewer tiles than the caller said)
                o = blk = i = t = t1 = left = 0;
                return true;
            }
            const int k = blk + lane;
            bool any = false;
            for (int g = 0; g < (w.patterns == w.batch * w.heads ? w.group : 1) && !any; ++g) {
                const int p = w.pattern(o, g);
                any = k < w.NB && w.at(p, k + 1) > w.at(p, k);
            }
            const unsigned found = __ballot_sync(~0u, any);
            if (found) {
                blk += __ffs(found) - 1;
                break;
            }
            blk = min(blk + 32, w.NB);
        }
        for (i = 0;; ++i) {
            const int p = w.pattern(o, i);
            t = w.at(p, blk);
            t1 = w.at(p, blk + 1);
            if (t < t1) break;
        }
        return true;
    }
};

template <typename T> struct GradArgsOf {
    TileArgsOf<T> a;
    Tiles w;
    const int *tile_at;       // of a tile: its row or column block, the first of two ints for dK and dV
    int share, ctas;          // cost of a CTA's blocks and tiles; CTAs
    const int4 *starts;       // of the CTAs: where their first tile lies
    const long long *first;   // its number, and that of the one behind the last CTA's
    float *part;              // [ctas][2][dK: 2][128][DP]
    int *bad;                 // [outers][blocks]: the sums of a block are not finite (its rows are taken one by one)
    // The first and the last CTA that have tiles of a block (c1 < c0: it has none); returns their number.
    __device__ __forceinline__ long long holders(int o, int blk, int &c0, int &c1) const
    {
        const long long ahead = w.ahead(o, blk), n = w.ahead(o, blk + 1) - ahead;
        const long long p0 = w.base(o) + ahead + (long long)w.per * ((long long)o * w.NB + blk + 1);
        c0 = (int)(p0 / share);
        c1 = n ? (int)((p0 + n - 1) / share) : c0 - 1;
        return n;
    }
};
using GradArgs = GradArgsOf<Bf16>;

// Two warps issue products: one S and dP, as far ahead as sets of tensor memory are free, one the second products.  The tensor core takes
// products from them in turn (about 52 cycles each at 128 x 64 x 16 from shared memory, 61 at 128 x 128 x 16 with A in tensor memory), and what
// a warp spends between its batches -- 100 to 250 cycles a barrier -- is hidden by the other's; with one issuer it was idle 44% of the time.
// 8 x 4096 x 4096 at 20%, width 64: 207 us with one issuer and a CTA per block, 193 us now; 16 heads over 4 of 8192, width 128, window
// of 1024 and 64 keys that all see: 677 us, with shares (the 64 keys' column block is as long as 64 others), two issuers and one join 339 us, and with blocks
// counted as two tiles more 322 us.
template <int MODE, int DP> struct GradCfg {
    static constexpr int SETS = MODE == kDkv && DP == 128 ? 2 : 3, THREADS = 256 * SETS + 96;
    static constexpr int STAGES = DP == 64 ? 6 : 4;
    static constexpr int ACCS = MODE == kDkv ? 2 : 1;
    static constexpr int TILE = 128 * DP * 2, HALF = 64 * DP * 2, STAT = MODE == kDkv ? 512 : 0;
    static constexpr int X1 = 0, X2 = TILE, Y1 = 2 * TILE, Y2 = Y1 + STAGES * HALF, ST = Y2 + STAGES * HALF, BAR = ST + STAGES * STAT, BYTES = BAR + 512 + 1024;
    static constexpr uint32_t COL_S = ACCS * DP, COLS = 512;   // accumulators (dQ, or dK and dV) first; S and dP of set i: COL_S + 128 i
    static_assert(COL_S + 128 * SETS <= 512 && BYTES <= 232448, "tensor memory or shared memory");
};
constexpr uint32_t kStepFirst = 1, kStepLast = 2;   // what the loading warp says of a step: its block's first, its block's last here

template <int MODE, int DP>
__global__ void __launch_bounds__(GradCfg<MODE, DP>::THREADS, 1)
tile_grad_kernel(const __grid_constant__ CUtensorMap tm_x1, const __grid_constant__ CUtensorMap tm_x2, const __grid_constant__ CUtensorMap tm_y1,
                 const __grid_constant__ CUtensorMap tm_y2, const __grid_constant__ GradArgs g)
{
    using C = GradCfg<MODE, DP>;
    constexpr int SETS = C::SETS, TMA_WARP = 8 * SETS, FIRST_WARP = TMA_WARP + 1, SECOND_WARP = TMA_WARP + 2;
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
    const TileArgs &a = g.a;
    const Shape &s = a.g.s;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) { ptx::mbar_init(full(i), 1); ptx::mbar_init(free_(i), 1); }
        for (int i = 0; i < SETS; ++i) { ptx::mbar_init(s_full(i), 1); ptx::mbar_init(p_full(i), 8); ptx::mbar_init(s_free(i), 1); }
        ptx::mbar_init(x_full, 1); ptx::mbar_init(x_free, 1); ptx::mbar_init(o_full, 1); ptx::mbar_init(o_free, 8 * SETS);
        ptx::mbar_init(slot + 16, 1); ptx::mbar_init(slot + 24, 1);   // the last products
        ptx::fence_mbar_init();
    }
    if (warp == FIRST_WARP) { ptx::tmem_alloc(slot, C::COLS); ptx::tmem_relinquish(); }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    asm volatile("griddepcontrol.wait;" ::: "memory");   // the row statistics and the shares' starts
    const uint32_t tmem = ptx::lds32(slot);
    const int tiles = (int)(g.first[blockIdx.x + 1] - g.first[blockIdx.x]), steps = 2 * tiles;
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {   // of a single thread
        if (ok && !wait_for(bar, parity)) { ok = false; *a.status = B2SP_ERR_TIMEOUT; }
        return ok;
    };
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return ok = __all_sync(~0u, wait(bar, parity)); };   // of a whole warp
    if (warp == TMA_WARP) {
        Walk w;
        w.start(g.w, g.starts[blockIdx.x], tiles);
        int i = 0, blocks = 0;
        for (bool more = tiles > 0; more && ok;) {
            const int b = w.o / g.w.outer, x = w.o % g.w.outer, h = x * g.w.group + w.i, hy = MODE == kDq ? h / (s.heads / s.kv_heads) : h, blk = w.blk;
            const int r0 = (MODE == kDq ? g.tile_at[w.t] : g.tile_at[2 * w.t]) * kTile;
            const bool fresh = w.fresh, last = w.next(g.w);
            more = w.left > 0;
            if (fresh) {   // the block's own operands, behind the last product that reads the previous block's
                if (!wait_all(x_free, (blocks & 1) ^ 1)) break;
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(x_full, 2 * C::TILE);
                    const Op &o1 = MODE == kDq ? a.q : a.k, &o2 = MODE == kDq ? a.dout : a.v;
                    load_tile<DP, 128>(base + C::X1, &tm_x1, x_full, blk * kTile, x * o1.hm, b * o1.bm);
                    load_tile<DP, 128>(base + C::X2, &tm_x2, x_full, blk * kTile, x * o2.hm, b * o2.bm);
                }
                __syncwarp();
                ++blocks;
            }
            for (int half = 0; half < 2; ++half, ++i) {
                const int st = i % C::STAGES, at = r0 + half * 64;
                if (!wait_all(free_(st), (i / C::STAGES & 1) ^ 1)) break;
                if (ptx::elect_one()) {
                    ptx::sts32(flags(st), (fresh && !half ? kStepFirst : 0) | (last && half ? kStepLast : 0));
                    ptx::mbar_arrive_expect_tx(full(st), 2 * C::HALF + C::STAT);
                    const Op &o1 = MODE == kDq ? a.k : a.q, &o2 = MODE == kDq ? a.v : a.dout;
                    load_tile<DP, 64>(base + C::Y1 + st * C::HALF, &tm_y1, full(st), at, hy * o1.hm, b * o1.bm);
                    load_tile<DP, 64>(base + C::Y2 + st * C::HALF, &tm_y2, full(st), at, hy * o2.hm, b * o2.bm);
                    if (MODE == kDkv) bulk_load(base + C::ST + st * C::STAT, a.g.stat + ((long long)b * s.heads + h) * a.g.stat_stride + at, C::STAT, full(st));
                }
                __syncwarp();
            }
        }
        // copies in flight land before the CTA ends, also where another warp gave up a wait
        if (blocks) ptx::mbar_wait(x_full, (blocks - 1) & 1);
        for (int k = max(0, i - C::STAGES); k < i; ++k) ptx::mbar_wait(full(k % C::STAGES), k / C::STAGES & 1);
    } else if (warp == FIRST_WARP) {
        if (ptx::elect_one()) {
            const int ks = (s.d + 15) >> 4;
            const uint32_t x1 = desc_columns(base + C::X1), x2 = desc_columns(base + C::X2), y1 = desc_columns(base + C::Y1), y2 = desc_columns(base + C::Y2);
            int st = 0, ph = 0, set = 0, round = 0, blocks = 0;
            for (int i = 0; i < steps; ++i) {
                if (!wait(full(st), ph)) break;
                if ((ptx::lds32(flags(st)) & kStepFirst) && !wait(x_full, blocks++ & 1)) break;
                if (round && !wait(s_free(set), (round - 1) & 1)) break;   // the second products of the step before last here are done
                const uint32_t to = tmem + C::COL_S + set * 128;
                product_columns<DP, 64>(to, x1, y1 + st * (C::HALF >> 4), ks);
                product_columns<DP, 64>(to + 64, x2, y2 + st * (C::HALF >> 4), ks);
                ptx::mma_commit(s_full(set));
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
            int st = 0, ph = 0, set = 0, round = 0, blocks = 0;
            bool onto = false;
            for (int i = 0; i < steps; ++i) {
                if (!wait(full(st), ph)) break;   // (long complete: what it says of the step is visible here)
                const uint32_t f = ptx::lds32(flags(st));
                if (f & kStepFirst) {
                    onto = false;
                    if (blocks && !wait(o_free, (blocks - 1) & 1)) break;   // the accumulators are read
                }
                if (!wait(p_full(set), round & 1)) break;
                ptx::tc_fence_after_sync();
                const uint32_t from = tmem + C::COL_S + set * 128;
                // (dQ: dS lies over S.  dK, dV: P over S, dS over dP.)
                if (MODE == kDkv) product_rows<DP, 64, 32>(tmem + DP, from, y2 + st * (C::HALF >> 4), onto);
                product_rows<DP, 64, 32>(tmem, from + (MODE == kDkv ? 64 : 0), y1 + st * (C::HALF >> 4), onto);
                onto = true;
                ptx::mma_commit(s_free(set));
                ptx::mma_commit(free_(st));
                if (f & kStepLast) {
                    ptx::mma_commit(x_free);
                    ptx::mma_commit(o_full);
                    ++blocks;
                }
                if (++st == C::STAGES) { st = 0; ph ^= 1; }
                if (++set == SETS) { set = 0; ++round; }
            }
            ptx::mma_commit(slot + 24);
            ptx::mbar_wait(slot + 24, 0);
        }
        __syncwarp();
    } else {
        const int set = warp >> 3, part = warp >> 2 & 1, lane_row = threadIdx.x & 127;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16), from = mine + C::COL_S + set * 128 + part * 32;
        const float c2 = s.scale * kLog2e;
        const uint64_t f2 = two(c2, c2);
        Walk w;
        w.start(g.w, g.starts[blockIdx.x], tiles);
        int i = 0, blocks = 0, at_set = 0, round = 0, st = 0;   // step, and which set, which of its turns and which stage it has
        float2 own = make_float2(0.f, 0.f);
        unsigned some = 0;
        int first_i = w.i, first_t = w.t;   // where the block's part began (is it the block's beginning?)
        for (bool more = tiles > 0; more && ok;) {
            const int blk = w.blk, o = w.o;
            if (w.fresh) {
                some = 0;
                first_i = w.i;
                first_t = w.t;
                if (MODE == kDq) own = a.g.stat[(long long)o * a.g.stat_stride + blk * kTile + lane_row];
            }
            const uint4 now = __ldg((MODE == kDq ? a.plan.masks : a.plan.tmasks) + (long long)w.t * kTile + lane_row);
            some |= now.x | now.y | now.z | now.w;
            const uint64_t l2 = two(own.x, own.x), d2 = two(own.y, own.y);
            for (int half = 0; half < 2; ++half, ++i) {
                const bool my_turn = at_set == set;
                const int stage = st, turn = round;
                if (++st == C::STAGES) st = 0;
                if (++at_set == SETS) { at_set = 0; ++round; }
                if (!my_turn) continue;
                if (!wait_all(s_full(set), turn & 1)) break;
                ptx::tc_fence_after_sync();
                const uint32_t stat = base + C::ST + stage * C::STAT + part * 256;
                const uint32_t m = half ? (part ? now.w : now.z) : (part ? now.y : now.x);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t x[16], y[16];
                    ptx::tmem_ld_32x16(from + 16 * c, x);
                    ptx::tmem_ld_32x16(from + 64 + 16 * c, y);
                    ptx::tmem_ld_wait();
                    settle(x);
                    settle(y);
                    uint32_t p[8], q[8];
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        float p0, p1, e0, e1;
                        uint64_t nl = l2, nd = d2;
                        if (MODE == kDkv) {
                            float l0, d0, l1, d1;
                            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(l0), "=f"(d0), "=f"(l1), "=f"(d1) : "r"(stat + (16 * c + k) * 8));
                            nl = two(l0, l1);
                            nd = two(d0, d1);
                        }
                        split(fma2(two(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), f2, nl), p0, p1);
                        p0 = m >> (16 * c + k) & 1 ? ex2(p0) : 0.f;
                        p1 = m >> (16 * c + k + 1) & 1 ? ex2(p1) : 0.f;
                        split(mul2(two(p0, p1), add2(two(__uint_as_float(y[k]), __uint_as_float(y[k + 1])), nd)), e0, e1);
                        if (MODE == kDkv) p[k >> 1] = bf16x2(p0, p1);
                        q[k >> 1] = bf16x2(e0, e1);
                    }
                    if (MODE == kDkv) {
                        tmem_st_32x8(from + 8 * c, p);
                        tmem_st_32x8(from + 64 + 8 * c, q);
                    } else {
                        tmem_st_32x8(from + 8 * c, q);
                    }
                }
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(p_full(set));   // (one arrival per warp: 32 on one word take turns)
            }
            const int last_i = w.i;
            const bool ended = w.t + 1 == w.t1;   // of the query head's tiles
            const bool ends = w.next(g.w);
            more = w.left > 0;
            if (!ends || !ok) continue;
            // the block's part is done: its sums leave tensor memory, the halves of the sets take the groups of 32 columns in turn
            if (!wait_all(o_full, blocks & 1)) break;
            ptx::tc_fence_after_sync();
            const int rows = MODE == kDq ? s.M : s.K, row = blk * kTile + lane_row;
            const int b = o / g.w.outer, h = o % g.w.outer;
            bool begun = true, whole = true;
            {
                // is the first tile here the block's first, the last one its last?
                for (int k = 0; k <= first_i; ++k) {
                    const int p = g.w.pattern(o, k), t0 = g.w.at(p, blk);
                    if (k < first_i ? g.w.at(p, blk + 1) > t0 : first_t > t0) begun = false;
                }
                whole = begun && ended;
                for (int k = last_i + 1; k < g.w.group && whole; ++k) {
                    const int p = g.w.pattern(o, k);
                    if (g.w.at(p, blk + 1) > g.w.at(p, blk)) whole = false;
                }
            }
            bool bad = false;
            const bool in = row < rows;
#pragma unroll 1
            for (int c = warp >> 2; c < C::ACCS * (DP / 32); c += 2 * SETS) {
                const int acc = c / (DP / 32), col = c % (DP / 32) * 32;
                uint32_t x[32];
                ptx::tmem_ld_32x32(mine + c * 32, x);
                ptx::tmem_ld_wait();
                settle(x);
                if (whole) {
                    Bf16 *to = (acc ? a.g.out2 : a.g.out1).at(b, h, in ? row : 0);
                    if (in && some) bad |= !store32(to, col, s.d, x, acc ? 1.f : s.scale);
                    else if (in)
                        for (int k = col; k < min(col + 32, s.d); k += 8) *reinterpret_cast<uint4 *>(to + k) = make_uint4(0, 0, 0, 0);
                } else {
                    float *to = g.part + ((((long long)blockIdx.x * 2 + begun) * C::ACCS + acc) * kTile + lane_row) * DP + col;
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        *reinterpret_cast<float4 *>(to + k) = make_float4(__uint_as_float(x[k]), __uint_as_float(x[k + 1]), __uint_as_float(x[k + 2]), __uint_as_float(x[k + 3]));
                }
            }
            if (bad) g.bad[(long long)o * g.w.NB + blk] = 1;
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(o_free);
            ++blocks;
        }
    }
    __syncwarp();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == FIRST_WARP) { ptx::tc_fence_after_sync(); ptx::tmem_dealloc(tmem, C::COLS); }
}

// Behind both passes of tile_grad_kernel.  Four CTAs of eight warps per share: if a block that begins in the share before goes on in this one, its
// parts are added up in order, 32 rows a CTA, a thread's up to eight groups of four elements at once; rows whose sums are not finite are taken one by
// one.  The CTAs also go through the flags of the blocks that were finished in one share.
constexpr int kJoinRows = 32, kJoinParts = kTile / kJoinRows;
template <int MODE, int DW, typename T, int V>
__device__ __forceinline__ void tile_grad_rows(const GradArgsOf<T> &g, int o, int blk, int r)
{
    const TileArgsOf<T> &a = g.a;
    const int b = o / g.w.outer, h = o % g.w.outer, row = blk * kTile + r;
    if (MODE == kDq) take_rows_again<kGradQ, DW, T, V>(a.g, a.g.ptr, a.g.idx, b, h, 1, row, 1u, a.g.ptr_stride, a.g.idx_stride);
    else take_rows_again<kGradKV, DW, T, V>(a.g, a.col_ptr, a.row_idx, b, h * g.w.group, g.w.group, row, 1u, a.g.s.K + 1ll, a.g.idx_stride);
}
// DP: columns of the sums; they are columns col0 and on of the outputs, dc of them.  DW: width class of whole rows.
template <int MODE, int DP, int DW, typename T, int V>
__device__ __forceinline__ void tile_grad_join(const GradArgsOf<T> &g, int cta, int ctas, int col0, int dc, int &redo)
{
    constexpr int ACCS = MODE == kDkv ? 2 : 1, LANES = ACCS * DP / 4, GROUPS = kJoinRows * LANES / 256;   // threads that a row takes; groups of a thread
    const TileArgsOf<T> &a = g.a;
    const Shape &s = a.g.s;
    const int share = cta / kJoinParts, part = cta % kJoinParts, warp = threadIdx.x >> 5;
    const int rows = MODE == kDq ? s.M : s.K;
    for (int block = cta; block < g.w.outers * g.w.NB; block += ctas)
        if (g.bad[block])
            for (int r = warp; r < kTile && block % g.w.NB * kTile + r < rows; r += 8) tile_grad_rows<MODE, DW, T, V>(g, block / g.w.NB, block % g.w.NB, r);
    if (share == 0 || g.first[share] == g.first[g.ctas]) return;
    const int4 at = g.starts[share];
    const int o = at.x, blk = at.y, b = o / g.w.outer, h = o % g.w.outer, row0 = blk * kTile + part * kJoinRows;
    int c0, c1;
    g.holders(o, blk, c0, c1);
    if (c0 != share - 1 || row0 >= rows) return;   // (the block begins with this share, or began before the last one)
    // four elements a group (of dK, then of dV)
    const int e = threadIdx.x % LANES * 4, acc = e / DP, col = e % DP, r0 = part * kJoinRows + threadIdx.x / LANES;
    const float *from = g.part + ((long long)acc * kTile + r0) * DP + col;
    float x[GROUPS][4] = {};
    for (int c = c0; c <= c1; ++c) {
        const float *p = from + ((long long)c * 2 + (c == c0)) * (ACCS * kTile * DP);
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const float4 v = *reinterpret_cast<const float4 *>(p + u * (256 / LANES) * DP);
            x[u][0] += v.x; x[u][1] += v.y; x[u][2] += v.z; x[u][3] += v.w;
        }
    }
    bool bad = false;
#pragma unroll
    for (int u = 0; u < GROUPS; ++u) {
        const int row = blk * kTile + r0 + u * (256 / LANES);
        if (row >= rows) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[u][k] *= acc ? 1.f : s.scale;
            bad |= col + k < dc && !(fabsf(x[u][k]) <= 3.402823466e38f);
        }
        store4<T, V>((acc ? a.g.out2 : a.g.out1).at(b, h, row) + col0, col, dc, x[u]);
    }
    if (bad) redo = 1;
    __syncthreads();
    if (redo == 0) return;
    for (int r = warp; r < kJoinRows && row0 + r < rows; r += 8) tile_grad_rows<MODE, DW, T, V>(g, o, blk, part * kJoinRows + r);
}
template <int DP, typename T = Bf16, int V = 4, int DW = DP>
__global__ void __launch_bounds__(256) tile_grad_join_kernel(const __grid_constant__ GradArgsOf<T> dq, const __grid_constant__ GradArgsOf<T> dkv, int col0, int dc)
{
    __shared__ int redo;
    const int first = dkv.ctas * kJoinParts, cta = blockIdx.x;   // (dK and dV first: they have the longer blocks)
    if (threadIdx.x == 0) redo = 0;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (cta < first) tile_grad_join<kDkv, DP, DW, T, V>(dkv, cta, first, col0, dc, redo);
    else tile_grad_join<kDq, DP, DW, T, V>(dq, cta - first, gridDim.x - first, col0, dc, redo);
}

// Ahead of both: row statistics (see attention_stat_kernel); and, in the first CTAs, where the shares begin, cleared flags of the blocks, and zeros for
// the blocks that have no tiles.
template <typename T> struct ShareArgsOf {
    Tiles w[2];
    int kinds;           // 1: only w[0]
    int share[2], ctas[2], rows[2];
    int4 *starts[2];
    long long *first[2], tiles[2];
    int *bad[2];         // NULL: neither flags nor zeros
    View<T> out[3];      // dQ, dK, dV
};
using ShareArgs = ShareArgsOf<Bf16>;
template <typename T> __device__ __forceinline__ void prepare_shares(const ShareArgsOf<T> &h, int d, int share_blocks)
{
    const int u = blockIdx.x * 256 + threadIdx.x, lane = threadIdx.x & 31, total = h.ctas[0] + (h.kinds > 1 ? h.ctas[1] : 0);
    for (int i = u; i < total + h.kinds; i += share_blocks * 256) {
        const int k = i <= h.ctas[0] ? 0 : 1, c = k ? i - h.ctas[0] - 1 : i;
        const long long first = c == h.ctas[k] ? h.tiles[k] : min(h.tiles[k], share_tile(h.w[k], (long long)c * h.share[k]));
        h.first[k][c] = first;
        if (c < h.ctas[k]) h.starts[k][c] = first < h.tiles[k] ? share_start(h.w[k], first) : make_int4(0, 0, 0, 0);
    }
    for (int k = 0; k < h.kinds; ++k) {
        const Tiles &w = h.w[k];
        if (!h.bad[k]) continue;
        for (int i0 = u - lane; i0 < w.outers * w.NB; i0 += share_blocks * 256) {
            const int i = i0 + lane, o = i / w.NB, blk = i % w.NB;
            bool none = false;
            if (i < w.outers * w.NB) {
                h.bad[k][i] = 0;
                none = w.ahead(o, blk + 1) == w.ahead(o, blk);
            }
            for (unsigned left = __ballot_sync(~0u, none); left; left &= left - 1) {
                const int z = i0 + __ffs(left) - 1, zo = z / w.NB, z0 = z % w.NB * kTile, n = min(kTile, h.rows[k] - z0);
                for (int e = lane; e < n * d; e += 32)
                    for (int x = k; x < (k ? 3 : 1); ++x) narrow(0.f, h.out[x].at(zo / w.outer, zo % w.outer, z0 + e / d)[e % d]);
            }
        }
    }
}
constexpr int kStatRows = 4;   // rows of half a warp
template <int DUMMY = 0>
__global__ void __launch_bounds__(256) tile_grad_stat_kernel(Shape s, View<const Bf16> out, View<const Bf16> dout, const float *lse, int stat_rows, float2 *stat,
                                                             const __grid_constant__ ShareArgs h, int share_blocks, int *status)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if ((int)blockIdx.x < share_blocks) {   // (first, as they wait longest)
        prepare_shares(h, s.d, share_blocks);
        return;
    }
    // half a warp per row, eight elements a lane, four rows at once
    const int half = threadIdx.x & 15, c = half * 8;
    const long long first = ((blockIdx.x - share_blocks) * 16ll + (threadIdx.x >> 4)) * kStatRows;   // (a problem has a multiple of 128 rows)
    const long long prob = first / stat_rows;
    if (prob >= (long long)s.batch * s.heads) return;
    const int row0 = (int)(first - prob * stat_rows), b = (int)(prob / s.heads), head = (int)(prob % s.heads);
    uint4 x[kStatRows], y[kStatRows];
    float top[kStatRows];
#pragma unroll
    for (int k = 0; k < kStatRows; ++k) {
        x[k] = y[k] = make_uint4(0, 0, 0, 0);
        top[k] = -CUDART_INF_F;
        if (row0 + k < s.M) {
            top[k] = lse[prob * s.M + row0 + k];
            if (c < s.d) {
                x[k] = __ldg(reinterpret_cast<const uint4 *>(out.at(b, head, row0 + k) + c));
                y[k] = __ldg(reinterpret_cast<const uint4 *>(dout.at(b, head, row0 + k) + c));
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kStatRows; ++k) {
        const unsigned u[4] = {x[k].x, x[k].y, x[k].z, x[k].w}, v[4] = {y[k].x, y[k].y, y[k].z, y[k].w};
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum = fmaf(__uint_as_float(u[i] << 16), __uint_as_float(v[i] << 16), sum);
            sum = fmaf(__uint_as_float(u[i] & 0xffff0000u), __uint_as_float(v[i] & 0xffff0000u), sum);
        }
#pragma unroll
        for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        if (half == 0) stat[first + k] = top[k] == -CUDART_INF_F ? make_float2(-CUDART_INF_F, 0.f) : make_float2(-top[k] * kLog2e, -sum);
    }
}

}  // namespace attn
}  // namespace b2sp
