// Attention over the tiles of a plan on the tensor cores (tcgen05, tensor memory, TMA): bfloat16, head widths up to 128.
//
// At the densities that masks have (10% to 30% scattered, or dense inside a window) a 128 x 128 tile of the pattern is cheaper multiplied
// whole than entry by entry: what is not stored is masked by the tile's 128 x 128 bits, which the plan holds ready.  Tiles without an entry are never
// visited.
//   forward  S = Q K^T into tensor memory; each thread of four softmax warps takes a row, masks, exponentiates, and writes the
//            weights back to tensor memory as bfloat16, over S; O += P V accumulates in tensor memory.
//   dQ       the same walk, S and dP = dO V^T side by side, ds = p (dp - delta) back as bfloat16, dQ += dS K.
//   dK, dV   a CTA per 128 keys walks the tiles of its column block, 64 queries at a time, with everything transposed (rows of
//            tensor memory are keys): dV += P^T dO, dK += dS^T Q, over all query heads that share the keys.
// Two passes over the tiles in the backward direction (seven products instead of five, the weights twice) need neither atomics nor a slab
// of fp32 gradients, so results are the same bits every time.
//
// What bounds them: the exponentials (16 a clock on an SM: 1024 clocks a tile) at width 64, together with the tensor core (two products of 512
// clocks a tile) at width 128.  Two CTAs per SM take turns between the two.
//
// The reference of the exponentials (the "maximum") is taken over all 128 products of a row's tile, masked or not, which spares the mask in
// that sweep; it moves only when it grows by more than 8 (to base 2), so O is rarely rescaled.  A row that loses its weights to
// a larger masked product (their sum below 2^-100), or meets a NaN or an infinity -- a masked weight of 0 times a row of V that holds one, which
// no entry names, is NaN -- is computed again entry by entry, by the row kernels' code.  Results are thus those of the stored entries alone.
#pragma once
#include <cuda.h>

#include "attention_tiles.h"
#include "ptx_sm100.cuh"

namespace b2sp {
namespace attn {

struct Op {              // a tensor map's coordinates of (b, h): 0 where the operand is shared
    int hm, bm;
};

struct TileArgs {
    RowArgs<Bf16> g;     // operands, pattern and outputs for rows that are taken one by one
    Plan plan;
    Op q, k, v, dout;
    const int *col_ptr, *row_idx;        // transposed pattern
    int *status;
};

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
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// After tmem_ld_wait(): nothing that uses the loaded registers moves in front of the wait.
__device__ __forceinline__ void settle(uint32_t (&x)[32])
{
    asm volatile("" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]), "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15]), "+r"(x[16]), "+r"(x[17]), "+r"(x[18]), "+r"(x[19]), "+r"(x[20]), "+r"(x[21]), "+r"(x[22]), "+r"(x[23]), "+r"(x[24]), "+r"(x[25]), "+r"(x[26]), "+r"(x[27]), "+r"(x[28]), "+r"(x[29]), "+r"(x[30]), "+r"(x[31]));
}

// Operand tiles in shared memory: blocks of 64 columns, each ROWS rows of 128 bytes, 128-byte swizzle.  The same bytes are an operand whose
// contraction runs along the columns (steps of 16: 32 bytes) or along the rows (steps of 16: 2 KB).
template <int ROWS> __device__ __forceinline__ uint64_t along_columns(uint32_t base, int step)
{
    return ptx::smem_desc_sw128(base + (step >> 2) * (ROWS * 128) + (step & 3) * 32, 16, 1024);
}
template <int ROWS> __device__ __forceinline__ uint64_t along_rows(uint32_t base, int step)
{
    return ptx::smem_desc_sw128(base + step * 2048, ROWS * 128, 1024);
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
template <int MODE, int DW>
__device__ __noinline__ void rows_one_by_one(const RowArgs<Bf16> &g, const int *ptr, const int *idx, int b, int h0, int heads, int row0, unsigned bad,
                                             long long ptr_stride, long long idx_stride)
{
    for (; bad; bad &= bad - 1) {
        const int row = row0 + __ffs(bad) - 1;
        RowWork<MODE, Bf16, 4, DW> w, all;
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

constexpr int kTileThreads = 192;   // four softmax warps, a TMA warp, an MMA warp

// ---- forward ---------------------------------------------------------------------------------------------------------------------
template <int DP> struct FwdCfg {
    static constexpr int STAGES = DP == 64 ? 2 : 1;
    static constexpr int TILE = 128 * DP * 2;
    static constexpr int Q = 0, K = TILE, V = K + STAGES * TILE, BAR = V + STAGES * TILE, BYTES = BAR + 256 + 1024;
    static constexpr uint32_t COL_S = 0, COL_O = 128, COLS = 256;
};

template <int DP>
__global__ void __launch_bounds__(kTileThreads, 2)
tile_forward_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ TileArgs a)
{
    using C = FwdCfg<DP>;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (ptx::smem_u32(raw) + 1023u) & ~1023u, bars = base + C::BAR;
    auto k_full = [&](int s) { return bars + 8u * s; };
    auto k_free = [&](int s) { return bars + 16u + 8u * s; };
    auto v_full = [&](int s) { return bars + 32u + 8u * s; };
    auto v_free = [&](int s) { return bars + 48u + 8u * s; };
    const uint32_t q_full = bars + 64, s_full = bars + 72, p_full = bars + 80, o_full = bars + 88, slot = bars + 96;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Shape &s = a.g.s;
    const int problems = s.batch * s.heads, RB = a.plan.RB;
    const int prob = blockIdx.x % problems, rb = RB - 1 - blockIdx.x / problems;   // (a causal mask's longest rows first)
    const int b = prob / s.heads, h = prob % s.heads, hkv = h / (s.heads / s.kv_heads);
    const int pat = pattern_of(s.patterns, s.batch, s.heads, b, h);
    const int t0 = a.plan.rb_ptr[pat * RB + rb], nt = a.plan.rb_ptr[pat * RB + rb + 1] - t0;
    const int row = rb * kTile + threadIdx.x;   // of a softmax thread
    float *lse = a.g.lse + (long long)prob * s.M;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
    if (nt == 0) {
        if (threadIdx.x < 128 && row < s.M) {
            Bf16 *o = a.g.out1.at(b, h, row);
            for (int c = 0; c < s.d; c += 8) *reinterpret_cast<uint4 *>(o + c) = make_uint4(0, 0, 0, 0);
            lse[row] = -CUDART_INF_F;
        }
        return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) {
            ptx::mbar_init(k_full(i), 1); ptx::mbar_init(k_free(i), 1);
            ptx::mbar_init(v_full(i), 1); ptx::mbar_init(v_free(i), 1);
        }
        ptx::mbar_init(q_full, 1); ptx::mbar_init(s_full, 1); ptx::mbar_init(p_full, 128); ptx::mbar_init(o_full, 1);
        ptx::fence_mbar_init();
    }
    if (warp == 5) { ptx::tmem_alloc(slot, C::COLS); ptx::tmem_relinquish(); }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = ptx::lds32(slot);
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !ptx::mbar_wait(bar, parity)) { ok = false; *a.status = B2SP_ERR_TIMEOUT; }
        return ok;
    };
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return ok = __all_sync(~0u, wait(bar, parity)); };   // of a softmax warp
    if (warp == 4) {
        if (ptx::elect_one()) {
            ptx::mbar_arrive_expect_tx(q_full, C::TILE);
            load_tile<DP, 128>(base + C::Q, &tm_q, q_full, rb * kTile, h * a.q.hm, b * a.q.bm);
            int i = 0, next = a.plan.tile_cb[t0];
            for (; i < nt; ++i) {
                const int st = i % C::STAGES, ph = i / C::STAGES & 1, cb = next;
                if (i + 1 < nt) next = a.plan.tile_cb[t0 + i + 1];
                if (!wait(k_free(st), ph ^ 1)) break;
                ptx::mbar_arrive_expect_tx(k_full(st), C::TILE);
                load_tile<DP, 128>(base + C::K + st * C::TILE, &tm_k, k_full(st), cb * kTile, hkv * a.k.hm, b * a.k.bm);
                if (!wait(v_free(st), ph ^ 1)) break;
                ptx::mbar_arrive_expect_tx(v_full(st), C::TILE);
                load_tile<DP, 128>(base + C::V + st * C::TILE, &tm_v, v_full(st), cb * kTile, hkv * a.v.hm, b * a.v.bm);
            }
            if (!ok) {   // copies in flight land before the CTA ends
                ptx::mbar_wait(q_full, 0);
                for (int k = max(0, i - C::STAGES); k <= i; ++k) { ptx::mbar_wait(k_full(k % C::STAGES), k / C::STAGES & 1); if (k < i) ptx::mbar_wait(v_full(k % C::STAGES), k / C::STAGES & 1); }
            }
        }
        __syncwarp();
    } else if (warp == 5) {
        if (ptx::elect_one()) {
            const int ks = (s.d + 15) >> 4;
            wait(q_full, 0);
            for (int i = 0; i < nt; ++i) {
                const int st = i % C::STAGES, ph = i / C::STAGES & 1;
                if (!wait(k_full(st), ph)) break;
                // (S of this tile overwrites the weights of the last: the tensor core takes its products in order)
                for (int k = 0; k < ks; ++k)
                    mma_ss(tmem + C::COL_S, along_columns<128>(base + C::Q, k), along_columns<128>(base + C::K + st * C::TILE, k), idesc_bf16(128, false), k > 0);
                ptx::mma_commit(k_free(st));
                ptx::mma_commit(s_full);
                if (!wait(p_full, i & 1) || !wait(v_full(st), ph)) break;
                ptx::tc_fence_after_sync();
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    mma_ts(tmem + C::COL_O, tmem + C::COL_S + k * 8, along_rows<128>(base + C::V + st * C::TILE, k), idesc_bf16(DP, true), (i | k) > 0);
                ptx::mma_commit(v_free(st));
            }
            ptx::mma_commit(o_full);
            if (!ok) ptx::mbar_wait(o_full, 0);   // products in flight end before tensor memory is freed
        }
        __syncwarp();
    } else {
        const float c2 = s.scale * kLog2e;
        const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16);
        const uint4 *mask = a.plan.masks + (long long)t0 * kTile + threadIdx.x;
        uint4 bits = __ldg(mask);
        float ref = 0.f;                       // reference of the exponentials, of the products before scaling
        uint64_t sums = two(0.f, 0.f);
        unsigned some = 0;
        for (int i = 0; i < nt; ++i) {
            const uint4 now = bits;
            if (i + 1 < nt) bits = __ldg(mask + (long long)(i + 1) * kTile);
            some |= now.x | now.y | now.z | now.w;
            if (!wait_all(s_full, i & 1)) break;
            ptx::tc_fence_after_sync();
            float top = -CUDART_INF_F;
            {
                uint32_t x[2][32];
                ptx::tmem_ld_32x32(mine + C::COL_S, x[0]);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    ptx::tmem_ld_wait();
                    settle(x[c & 1]);
                    if (c < 3) ptx::tmem_ld_32x32(mine + C::COL_S + 32 * (c + 1), x[(c + 1) & 1]);
#pragma unroll
                    for (int k = 0; k < 32; ++k) top = fmaxf(top, __uint_as_float(x[c & 1][k]));
                }
            }
            const bool move = i == 0 || (top - ref) * c2 > 8.f;
            if (__any_sync(~0u, move)) {
                const float to = top == -CUDART_INF_F ? 0.f : i == 0 ? top : fmaxf(top, ref), fall = i == 0 ? 0.f : ex2((ref - to) * c2);
                ref = to;
                sums = mul2(sums, two(fall, fall));
                if (i) {
                    const uint64_t f2 = two(fall, fall);
#pragma unroll 1
                    for (int c = 0; c < DP; c += 32) {
                        uint32_t x[32];
                        ptx::tmem_ld_32x32(mine + C::COL_O + c, x);
                        ptx::tmem_ld_wait();
                        settle(x);
#pragma unroll
                        for (int k = 0; k < 32; k += 2) {
                            float y0, y1;
                            split(mul2(two(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), f2), y0, y1);
                            x[k] = __float_as_uint(y0);
                            x[k + 1] = __float_as_uint(y1);
                        }
                        ptx::tmem_st_32x32(mine + C::COL_O + c, x);
                    }
                }
            }
            const uint64_t f2 = two(c2, c2), r2 = two(-ref * c2, -ref * c2);
            uint32_t x[2][32];
            ptx::tmem_ld_32x32(mine + C::COL_S, x[0]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                ptx::tmem_ld_wait();
                settle(x[c & 1]);
                if (c < 3) ptx::tmem_ld_32x32(mine + C::COL_S + 32 * (c + 1), x[(c + 1) & 1]);
                const uint32_t w = c == 0 ? now.x : c == 1 ? now.y : c == 2 ? now.z : now.w;
                uint32_t p[16];
#pragma unroll
                for (int k = 0; k < 32; k += 2) {
                    float y0, y1;
                    split(fma2(two(__uint_as_float(x[c & 1][k]), __uint_as_float(x[c & 1][k + 1])), f2, r2), y0, y1);
                    y0 = w >> k & 1 ? ex2(y0) : 0.f;
                    y1 = w >> (k + 1) & 1 ? ex2(y1) : 0.f;
                    sums = add2(sums, two(y0, y1));
                    p[k >> 1] = bf16x2(y0, y1);
                }
                ptx::tmem_st_32x16(mine + C::COL_S + 16 * c, p);   // over columns of S that are read already
            }
            ptx::tmem_st_wait();
            ptx::tc_fence_before_sync();
            ptx::mbar_arrive(p_full);
        }
        wait_all(o_full, 0);
        ptx::tc_fence_after_sync();
        float l, l1;
        split(sums, l, l1);
        l += l1;
        const bool in = row < s.M, live = in && some;
        bool bad = live && !(l >= 7.8886091e-31f && l <= 3.402823466e38f);
        const float inv = live ? 1.f / l : 0.f;
        Bf16 *o = a.g.out1.at(b, h, in ? row : 0);
#pragma unroll 1
        for (int c = 0; c < DP; c += 32) {
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
        if (redo && ok) rows_one_by_one<kForward, DP>(a.g, a.g.ptr, a.g.idx, b, h, 1, rb * kTile + warp * 32, redo, a.g.ptr_stride, a.g.idx_stride);
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 5) { ptx::tc_fence_after_sync(); ptx::tmem_dealloc(tmem, C::COLS); }
}

// ---- dQ --------------------------------------------------------------------------------------------------------------------------
// 64 keys a step.  (One stage of K and V at width 128: two CTAs per SM hold 96 KB each.)
template <int DP> struct DqCfg {
    static constexpr int STAGES = DP == 64 ? 3 : 1;
    static constexpr int TILE = 128 * DP * 2, HALF = 64 * DP * 2;
    static constexpr int Q = 0, DO = TILE, K = 2 * TILE, V = K + STAGES * HALF, BAR = V + STAGES * HALF, BYTES = BAR + 256 + 1024;
    static constexpr uint32_t COL_S = 0, COL_P = 64, COL_Q = 128, COLS = 256;
};

template <int DP>
__global__ void __launch_bounds__(kTileThreads, 2)
tile_dq_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_k,
               const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ TileArgs a)
{
    using C = DqCfg<DP>;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (ptx::smem_u32(raw) + 1023u) & ~1023u, bars = base + C::BAR;
    auto full = [&](int s) { return bars + 8u * s; };
    auto free_ = [&](int s) { return bars + 32u + 8u * s; };
    const uint32_t q_full = bars + 64, s_full = bars + 72, p_full = bars + 80, o_full = bars + 88, slot = bars + 96;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Shape &s = a.g.s;
    const int problems = s.batch * s.heads, RB = a.plan.RB;
    const int prob = blockIdx.x % problems, rb = RB - 1 - blockIdx.x / problems;
    const int b = prob / s.heads, h = prob % s.heads, hkv = h / (s.heads / s.kv_heads);
    const int pat = pattern_of(s.patterns, s.batch, s.heads, b, h);
    const int t0 = a.plan.rb_ptr[pat * RB + rb], steps = 2 * (a.plan.rb_ptr[pat * RB + rb + 1] - t0);
    const int row = rb * kTile + threadIdx.x;
    if (steps == 0) {
        if (threadIdx.x < 128 && row < s.M) {
            Bf16 *o = a.g.out1.at(b, h, row);
            for (int c = 0; c < s.d; c += 8) *reinterpret_cast<uint4 *>(o + c) = make_uint4(0, 0, 0, 0);
        }
        return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) { ptx::mbar_init(full(i), 1); ptx::mbar_init(free_(i), 1); }
        ptx::mbar_init(q_full, 1); ptx::mbar_init(s_full, 1); ptx::mbar_init(p_full, 128); ptx::mbar_init(o_full, 1);
        ptx::fence_mbar_init();
    }
    if (warp == 5) { ptx::tmem_alloc(slot, C::COLS); ptx::tmem_relinquish(); }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = ptx::lds32(slot);
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !ptx::mbar_wait(bar, parity)) { ok = false; *a.status = B2SP_ERR_TIMEOUT; }
        return ok;
    };
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return ok = __all_sync(~0u, wait(bar, parity)); };   // of a softmax warp
    if (warp == 4) {
        if (ptx::elect_one()) {
            ptx::mbar_arrive_expect_tx(q_full, 2 * C::TILE);
            load_tile<DP, 128>(base + C::Q, &tm_q, q_full, rb * kTile, h * a.q.hm, b * a.q.bm);
            load_tile<DP, 128>(base + C::DO, &tm_do, q_full, rb * kTile, h * a.dout.hm, b * a.dout.bm);
            int i = 0, now = 0, next = a.plan.tile_cb[t0];
            for (; i < steps; ++i) {
                if (!(i & 1)) {
                    now = next * kTile;
                    if (i + 2 < steps) next = a.plan.tile_cb[t0 + (i >> 1) + 1];
                }
                const int st = i % C::STAGES, ph = i / C::STAGES & 1, at = now + (i & 1) * 64;
                if (!wait(free_(st), ph ^ 1)) break;
                ptx::mbar_arrive_expect_tx(full(st), 2 * C::HALF);
                load_tile<DP, 64>(base + C::K + st * C::HALF, &tm_k, full(st), at, hkv * a.k.hm, b * a.k.bm);
                load_tile<DP, 64>(base + C::V + st * C::HALF, &tm_v, full(st), at, hkv * a.v.hm, b * a.v.bm);
            }
            if (!ok) {
                ptx::mbar_wait(q_full, 0);
                for (int k = max(0, i - C::STAGES); k < i; ++k) ptx::mbar_wait(full(k % C::STAGES), k / C::STAGES & 1);
            }
        }
        __syncwarp();
    } else if (warp == 5) {
        if (ptx::elect_one()) {
            const int ks = (s.d + 15) >> 4;
            wait(q_full, 0);
            for (int i = 0; i < steps; ++i) {
                const int st = i % C::STAGES, ph = i / C::STAGES & 1;
                const uint32_t K = base + C::K + st * C::HALF, V = base + C::V + st * C::HALF;
                if (!wait(full(st), ph)) break;
                for (int k = 0; k < ks; ++k) mma_ss(tmem + C::COL_S, along_columns<128>(base + C::Q, k), along_columns<64>(K, k), idesc_bf16(64, false), k > 0);
                for (int k = 0; k < ks; ++k) mma_ss(tmem + C::COL_P, along_columns<128>(base + C::DO, k), along_columns<64>(V, k), idesc_bf16(64, false), k > 0);
                ptx::mma_commit(s_full);
                if (!wait(p_full, i & 1)) break;
                ptx::tc_fence_after_sync();
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    mma_ts(tmem + C::COL_Q, tmem + C::COL_S + k * 8, along_rows<64>(K, k), idesc_bf16(DP, true), (i | k) > 0);
                ptx::mma_commit(free_(st));
            }
            ptx::mma_commit(o_full);
            if (!ok) ptx::mbar_wait(o_full, 0);   // products in flight end before tensor memory is freed
        }
        __syncwarp();
    } else {
        const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16);
        const float2 st = a.g.stat[(long long)prob * a.g.stat_stride + row];
        const float c2 = s.scale * kLog2e;
        const uint64_t f2 = two(c2, c2), l2 = two(-st.x, -st.x), d2 = two(-st.y, -st.y);
        const uint4 *mask = a.plan.masks + (long long)t0 * kTile + threadIdx.x;
        uint4 bits = __ldg(mask), now = bits;
        unsigned some = 0;
        for (int i = 0; i < steps; ++i) {
            if (!(i & 1)) {
                now = bits;
                some |= now.x | now.y | now.z | now.w;
                if (i + 2 < steps) bits = __ldg(mask + (long long)((i >> 1) + 1) * kTile);
            }
            if (!wait_all(s_full, i & 1)) break;
            ptx::tc_fence_after_sync();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t x[32], y[32];
                ptx::tmem_ld_32x32(mine + C::COL_S + 32 * c, x);
                ptx::tmem_ld_32x32(mine + C::COL_P + 32 * c, y);
                ptx::tmem_ld_wait();
                settle(x);
                settle(y);
                const uint32_t w = (i & 1) ? (c ? now.w : now.z) : (c ? now.y : now.x);
                uint32_t o[16];
#pragma unroll
                for (int k = 0; k < 32; k += 2) {
                    float p0, p1, e0, e1;
                    split(fma2(two(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), f2, l2), p0, p1);
                    split(mul2(two(ex2(p0), ex2(p1)), add2(two(__uint_as_float(y[k]), __uint_as_float(y[k + 1])), d2)), e0, e1);
                    o[k >> 1] = bf16x2(w >> k & 1 ? e0 : 0.f, w >> (k + 1) & 1 ? e1 : 0.f);
                }
                ptx::tmem_st_32x16(mine + C::COL_S + 16 * c, o);
            }
            ptx::tmem_st_wait();
            ptx::tc_fence_before_sync();
            ptx::mbar_arrive(p_full);
        }
        wait_all(o_full, 0);
        ptx::tc_fence_after_sync();
        const bool in = row < s.M, live = in && some;
        bool bad = false;
        Bf16 *o = a.g.out1.at(b, h, in ? row : 0);
#pragma unroll 1
        for (int c = 0; c < DP; c += 32) {
            uint32_t x[32];
            ptx::tmem_ld_32x32(mine + C::COL_Q + c, x);
            ptx::tmem_ld_wait();
            settle(x);
            if (live) bad |= !store32(o, c, s.d, x, s.scale);
            else if (in)
                for (int k = c; k < min(c + 32, s.d); k += 8) *reinterpret_cast<uint4 *>(o + k) = make_uint4(0, 0, 0, 0);
        }
        const unsigned redo = __ballot_sync(~0u, bad);
        if (redo && ok) rows_one_by_one<kGradQ, DP>(a.g, a.g.ptr, a.g.idx, b, h, 1, rb * kTile + warp * 32, redo, a.g.ptr_stride, a.g.idx_stride);
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 5) { ptx::tc_fence_after_sync(); ptx::tmem_dealloc(tmem, C::COLS); }
}

// ---- dK and dV -------------------------------------------------------------------------------------------------------------------
// Steps of 64 queries.  Width 64: two CTAs per SM, one set of four softmax warps each.  Width 128 fills tensor memory with the two
// accumulators and two sets of S and dP, so one CTA per SM has two sets of warps that take alternate steps.
template <int DP> struct DkvCfg {
    static constexpr int SETS = DP == 64 ? 1 : 2, THREADS = 128 * SETS + 64;
    static constexpr int STAGES = DP == 64 ? 3 : 3;
    static constexpr int TILE = 128 * DP * 2, HALF = 64 * DP * 2, STAT = 512;
    static constexpr int K = 0, V = TILE, Q = 2 * TILE, DO = Q + STAGES * HALF, ST = DO + STAGES * HALF, BAR = ST + STAGES * STAT, BYTES = BAR + 256 + 1024;
    static constexpr uint32_t COL_V = 0, COL_K = DP, COL_S = 2 * DP, COLS = DP == 64 ? 256 : 512;   // S and dP of set i: COL_S + 128 i
};

template <int DP>
__global__ void __launch_bounds__(DkvCfg<DP>::THREADS, DP == 64 ? 2 : 1)
tile_dkv_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_k,
                const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ TileArgs a)
{
    using C = DkvCfg<DP>;
    constexpr int SETS = C::SETS, TMA_WARP = 4 * SETS, MMA_WARP = TMA_WARP + 1;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (ptx::smem_u32(raw) + 1023u) & ~1023u, bars = base + C::BAR;
    auto full = [&](int s) { return bars + 8u * s; };
    auto free_ = [&](int s) { return bars + 32u + 8u * s; };
    auto s_full = [&](int w) { return bars + 64u + 8u * w; };
    auto p_full = [&](int w) { return bars + 80u + 8u * w; };
    const uint32_t k_full = bars + 96, o_full = bars + 104, slot = bars + 112;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Shape &s = a.g.s;
    const int CB = a.plan.CB, group = s.heads / s.kv_heads, problems = s.batch * s.kv_heads;
    const int prob = blockIdx.x % problems, cb = blockIdx.x / problems;
    const int b = prob / s.kv_heads, hkv = prob % s.kv_heads;
    // the walk: query heads of the group, tiles of the column block, halves of a tile
    int steps = 0;
    for (int i = 0; i < group; ++i) {
        const int pat = pattern_of(s.patterns, s.batch, s.heads, b, hkv * group + i);
        steps += 2 * (a.plan.cb_ptr[pat * CB + cb + 1] - a.plan.cb_ptr[pat * CB + cb]);
    }
    const int key = cb * kTile + (threadIdx.x & 127);
    if (steps == 0) {
        if (threadIdx.x < 128 && key < s.K) {
            Bf16 *o1 = a.g.out1.at(b, hkv, key), *o2 = a.g.out2.at(b, hkv, key);
            for (int c = 0; c < s.d; c += 8) *reinterpret_cast<uint4 *>(o1 + c) = *reinterpret_cast<uint4 *>(o2 + c) = make_uint4(0, 0, 0, 0);
        }
        return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) { ptx::mbar_init(full(i), 1); ptx::mbar_init(free_(i), 1); }
        for (int i = 0; i < SETS; ++i) { ptx::mbar_init(s_full(i), 1); ptx::mbar_init(p_full(i), 128); }
        ptx::mbar_init(k_full, 1); ptx::mbar_init(o_full, 1);
        ptx::fence_mbar_init();
    }
    if (warp == MMA_WARP) { ptx::tmem_alloc(slot, C::COLS); ptx::tmem_relinquish(); }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = ptx::lds32(slot);
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !ptx::mbar_wait(bar, parity)) { ok = false; *a.status = B2SP_ERR_TIMEOUT; }
        return ok;
    };
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return ok = __all_sync(~0u, wait(bar, parity)); };   // of a softmax warp
    if (warp == TMA_WARP) {
        if (ptx::elect_one()) {
            ptx::mbar_arrive_expect_tx(k_full, 2 * C::TILE);
            load_tile<DP, 128>(base + C::K, &tm_k, k_full, cb * kTile, hkv * a.k.hm, b * a.k.bm);
            load_tile<DP, 128>(base + C::V, &tm_v, k_full, cb * kTile, hkv * a.v.hm, b * a.v.bm);
            int i = 0;
            for (int hh = 0; hh < group && ok; ++hh) {
                const int h = hkv * group + hh, pat = pattern_of(s.patterns, s.batch, s.heads, b, h);
                const float2 *stat = a.g.stat + ((long long)b * s.heads + h) * a.g.stat_stride;
                const int t1 = a.plan.cb_ptr[pat * CB + cb + 1];
                for (int t = a.plan.cb_ptr[pat * CB + cb]; t < t1 && ok; ++t) {
                    const int r0 = a.plan.ctile[t].x * kTile;
                    for (int half = 0; half < 2; ++half, ++i) {
                        const int st = i % C::STAGES, ph = i / C::STAGES & 1, at = r0 + half * 64;
                        if (!wait(free_(st), ph ^ 1)) break;
                        ptx::mbar_arrive_expect_tx(full(st), 2 * C::HALF + C::STAT);
                        load_tile<DP, 64>(base + C::Q + st * C::HALF, &tm_q, full(st), at, h * a.q.hm, b * a.q.bm);
                        load_tile<DP, 64>(base + C::DO + st * C::HALF, &tm_do, full(st), at, h * a.dout.hm, b * a.dout.bm);
                        bulk_load(base + C::ST + st * C::STAT, stat + at, C::STAT, full(st));
                    }
                }
            }
            if (!ok) {
                ptx::mbar_wait(k_full, 0);
                for (int k = max(0, i - C::STAGES); k < i; ++k) ptx::mbar_wait(full(k % C::STAGES), k / C::STAGES & 1);
            }
        }
        __syncwarp();
    } else if (warp == MMA_WARP) {
        if (ptx::elect_one()) {
            const int ks = (s.d + 15) >> 4;
            auto first = [&](int i) {   // S^T and dP^T of step i
                const int st = i % C::STAGES;
                if (!wait(full(st), i / C::STAGES & 1)) return;
                const uint32_t to = tmem + C::COL_S + (i % SETS) * 128;
                for (int k = 0; k < ks; ++k) mma_ss(to, along_columns<128>(base + C::K, k), along_columns<64>(base + C::Q + st * C::HALF, k), idesc_bf16(64, false), k > 0);
                for (int k = 0; k < ks; ++k) mma_ss(to + 64, along_columns<128>(base + C::V, k), along_columns<64>(base + C::DO + st * C::HALF, k), idesc_bf16(64, false), k > 0);
                ptx::mma_commit(s_full(i % SETS));
            };
            wait(k_full, 0);
            for (int i = 0; i < SETS && i < steps; ++i) first(i);
            for (int i = 0; i < steps && ok; ++i) {
                const int st = i % C::STAGES;
                const uint32_t from = tmem + C::COL_S + (i % SETS) * 128;
                if (!wait(p_full(i % SETS), i / SETS & 1)) break;
                ptx::tc_fence_after_sync();
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_ts(tmem + C::COL_V, from + k * 8, along_rows<64>(base + C::DO + st * C::HALF, k), idesc_bf16(DP, true), (i | k) > 0);
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_ts(tmem + C::COL_K, from + 64 + k * 8, along_rows<64>(base + C::Q + st * C::HALF, k), idesc_bf16(DP, true), (i | k) > 0);
                ptx::mma_commit(free_(st));
                if (i + SETS < steps) first(i + SETS);
            }
            ptx::mma_commit(o_full);
            if (!ok) ptx::mbar_wait(o_full, 0);   // products in flight end before tensor memory is freed
        }
        __syncwarp();
    } else {
        const int set = SETS == 1 ? 0 : warp >> 2;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16), from = mine + C::COL_S + set * 128;
        const float c2 = s.scale * kLog2e;
        const uint64_t f2 = two(c2, c2);
        unsigned some = 0;
        int i = 0;
        for (int hh = 0; hh < group && ok; ++hh) {
            const int h = hkv * group + hh, pat = pattern_of(s.patterns, s.batch, s.heads, b, h);
            const int t1 = a.plan.cb_ptr[pat * CB + cb + 1];
            for (int t = a.plan.cb_ptr[pat * CB + cb]; t < t1 && ok; ++t) {
                const uint4 now = __ldg(a.plan.tmasks + (long long)t * kTile + (threadIdx.x & 127));
                some |= now.x | now.y | now.z | now.w;
                for (int half = 0; half < 2; ++half, ++i) {
                    if (SETS == 2 && (i & 1) != set) continue;
                    if (!wait_all(s_full(set), i / SETS & 1)) break;
                    ptx::tc_fence_after_sync();
                    const uint32_t stat = base + C::ST + (i % C::STAGES) * C::STAT;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t x[32], y[32];
                        ptx::tmem_ld_32x32(from + 32 * c, x);
                        ptx::tmem_ld_32x32(from + 64 + 32 * c, y);
                        ptx::tmem_ld_wait();
                        settle(x);
                        settle(y);
                        const uint32_t w = half ? (c ? now.w : now.z) : (c ? now.y : now.x);
                        uint32_t p[16], o[16];
#pragma unroll
                        for (int k = 0; k < 32; k += 2) {
                            float l0, d0, l1, d1, p0, p1, e0, e1;
                            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(l0), "=f"(d0), "=f"(l1), "=f"(d1) : "r"(stat + (32 * c + k) * 8));
                            split(fma2(two(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), f2, two(-l0, -l1)), p0, p1);
                            p0 = w >> k & 1 ? ex2(p0) : 0.f;
                            p1 = w >> (k + 1) & 1 ? ex2(p1) : 0.f;
                            split(mul2(two(p0, p1), add2(two(__uint_as_float(y[k]), __uint_as_float(y[k + 1])), two(-d0, -d1))), e0, e1);
                            p[k >> 1] = bf16x2(p0, p1);
                            o[k >> 1] = bf16x2(e0, e1);
                        }
                        ptx::tmem_st_32x16(from + 16 * c, p);
                        ptx::tmem_st_32x16(from + 64 + 16 * c, o);
                    }
                    ptx::tmem_st_wait();
                    ptx::tc_fence_before_sync();
                    ptx::mbar_arrive(p_full(set));
                }
            }
        }
        wait_all(o_full, 0);
        ptx::tc_fence_after_sync();
        const bool in = key < s.K, live = in && some;
        bool bad = false;
#pragma unroll 1
        for (int which = SETS == 2 ? set : 0; which < (SETS == 2 ? set + 1 : 2); ++which) {   // dV, dK
            Bf16 *o = which ? a.g.out1.at(b, hkv, in ? key : 0) : a.g.out2.at(b, hkv, in ? key : 0);
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
                uint32_t x[32];
                ptx::tmem_ld_32x32(mine + (which ? C::COL_K : C::COL_V) + c, x);
                ptx::tmem_ld_wait();
                settle(x);
                if (live) bad |= !store32(o, c, s.d, x, which ? s.scale : 1.f);
                else if (in)
                    for (int k = c; k < min(c + 32, s.d); k += 8) *reinterpret_cast<uint4 *>(o + k) = make_uint4(0, 0, 0, 0);
            }
        }
        if (SETS == 2) {   // a column of either gradient that is not finite: both are computed again, by the second set, after both are stored
            uint32_t *flag = reinterpret_cast<uint32_t *>(raw) + ((base + C::BAR + 128 - ptx::smem_u32(raw)) >> 2);   // one word per warp of the first set
            const unsigned vote = __ballot_sync(~0u, bad);
            if (set == 0 && lane == 0) flag[warp] = vote;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (set == 1) {
                const unsigned redo = vote | flag[warp & 3];
                if (redo && ok) rows_one_by_one<kGradKV, DP>(a.g, a.col_ptr, a.row_idx, b, hkv * group, group, cb * kTile + (warp & 3) * 32, redo, s.K + 1ll, a.g.idx_stride);
            }
        } else {
            const unsigned redo = __ballot_sync(~0u, bad);
            if (redo && ok) rows_one_by_one<kGradKV, DP>(a.g, a.col_ptr, a.row_idx, b, hkv * group, group, cb * kTile + warp * 32, redo, s.K + 1ll, a.g.idx_stride);
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == MMA_WARP) { ptx::tc_fence_after_sync(); ptx::tmem_dealloc(tmem, C::COLS); }
}

}  // namespace attn
}  // namespace b2sp
