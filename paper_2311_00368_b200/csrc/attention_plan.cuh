// Analysis of a mask for attention: what the tensor-core kernels and the backward pass need to know of a CSR pattern, found
// once for all calls on it.
//
// The pattern is cut into 128 x 128 tiles.  A plan lists the tiles that hold an entry, row block by row block (the order of
// the forward pass and of dQ) and column block by column block (dK and dV), each with its 128 x 128 bits in both orientations
// (2 KB each; a tile of the CSR arrays at 20% density is 13 KB), and the transposed pattern (col_ptr, row_idx; rows ascending)
// for the row kernels.  Every part is a function of the pattern alone: counters are integers, places come from ranks, never from the
// order in which atomics arrive.  A column out of range is left out and reported through the plan's flag word, as is a column that
// a row stores twice.
#pragma once
#include "attention.h"

namespace b2sp {
namespace attn {

struct Csr {
    const int *row_ptr, *col_idx;
    long long rp_stride, nz_stride;
    int M, K;
};

// The entry range of a pattern's rows [r0, r1), held inside the arrays whatever row_ptr says.
__device__ __forceinline__ void entry_range(const int *rp, long long nnz, int r0, int r1, int &a, int &e)
{
    const int most = (int)(nnz < 0x7fffffff ? nnz : 0x7fffffff);
    a = min(max(rp[r0], 0), most);
    e = min(max(rp[r1], a), most);
}

// One CTA per (pattern, row block): which column blocks it touches, and how many.
__global__ void plan_mark_kernel(Csr s, int RB, int CB, int words, unsigned *bitmap, unsigned *rank, int *count, unsigned long long *total,
                                 int *flags)
{
    extern __shared__ unsigned bits[];
    __shared__ int sums[32];
    const int p = blockIdx.x / RB, rb = blockIdx.x % RB;
    const int *rp = s.row_ptr + p * s.rp_stride, *ci = s.col_idx + p * s.nz_stride;
    for (int w = threadIdx.x; w < words; w += blockDim.x) bits[w] = 0;
    __syncthreads();
    int a, e;
    entry_range(rp, s.nz_stride, rb * kTile, min(s.M, rb * kTile + kTile), a, e);
    bool bad = false;
    for (long long i = a + (long long)threadIdx.x; i < e; i += blockDim.x) {
        const unsigned j = (unsigned)ci[i];
        if (j < (unsigned)s.K) {
            const unsigned cb = j / kTile, m = 1u << (cb & 31);
            if (!(bits[cb >> 5] & m)) atomicOr(&bits[cb >> 5], m);
        } else {
            bad = true;
        }
    }
    if (bad) atomicOr(flags, kPlanBadColumn);
    if (threadIdx.x < 32 && rb == 0 && threadIdx.x == 0 && rp[0] != 0) atomicOr(flags, kPlanBadColumn);
    for (int r = rb * kTile + threadIdx.x; r < min(s.M, rb * kTile + kTile); r += blockDim.x)
        if (rp[r + 1] < rp[r] || rp[r + 1] > s.nz_stride) atomicOr(flags, kPlanBadColumn);
    __syncthreads();
    // exclusive ranks of the words: chunks of blockDim.x words, a running base
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    int base = 0;
    for (int w0 = 0; w0 < words; w0 += blockDim.x) {
        const int w = w0 + threadIdx.x;
        const int c = w < words ? __popc(bits[w]) : 0;
        int x = c;
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(~0u, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) sums[warp] = x;
        __syncthreads();
        int before = base, all = 0;
        for (int k = 0; k < nw; ++k) {
            if (k < warp) before += sums[k];
            all += sums[k];
        }
        if (w < words && bitmap) {
            bitmap[(size_t)blockIdx.x * words + w] = bits[w];
            rank[(size_t)blockIdx.x * words + w] = before + x - c;
        }
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        if (count) count[blockIdx.x] = base;
        if (total) atomicAdd(total, (unsigned long long)base);
    }
}

// Exclusive scan of n counts in place, the total behind them; one CTA of 1024 threads.  blockIdx.x: independent arrays `stride` apart.
__global__ void plan_scan_kernel(int *v, long long n, long long stride)
{
    __shared__ int sums[32];
    v += blockIdx.x * stride;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int base = 0;
    constexpr int PER = 8;
    for (long long i0 = 0; i0 < n; i0 += 1024 * PER) {
        const long long i = i0 + (long long)threadIdx.x * PER;
        int c[PER], mine = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            c[k] = i + k < n ? v[i + k] : 0;
            mine += c[k];
        }
        int x = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(~0u, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) sums[warp] = x;
        __syncthreads();
        int at = base + x - mine, all = 0;
        for (int k = 0; k < 32; ++k) {
            if (k < warp) at += sums[k];
            all += sums[k];
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (i + k < n) v[i + k] = at;
            at += c[k];
        }
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) v[n] = base;
}

// One thread per (pattern, column block): how many row blocks touch it.
__global__ void plan_column_count_kernel(int P, int RB, int CB, int words, const unsigned *bitmap, int *count)
{
    const long long i = blockIdx.x * (long long)blockDim.x + threadIdx.x;
    if (i >= (long long)P * CB) return;
    const int p = (int)(i / CB), cb = (int)(i % CB);
    int n = 0;
    for (int rb = 0; rb < RB; ++rb) n += bitmap[((size_t)p * RB + rb) * words + (cb >> 5)] >> (cb & 31) & 1;
    count[i] = n;
}

// One thread per (pattern, column block): its tiles in the order of the row blocks.
__global__ void plan_column_list_kernel(int P, int RB, int CB, int words, const unsigned *bitmap, const unsigned *rank, const int *rb_ptr,
                                        const int *cb_ptr, long long tiles, int2 *ctile, int *tile_cb)
{
    const long long i = blockIdx.x * (long long)blockDim.x + threadIdx.x;
    if (i >= (long long)P * CB) return;
    const int p = (int)(i / CB), cb = (int)(i % CB);
    long long at = cb_ptr[i];
    for (int rb = 0; rb < RB; ++rb) {
        const size_t row = (size_t)p * RB + rb, w = row * words + (cb >> 5);
        const unsigned b = bitmap[w];
        if (!(b >> (cb & 31) & 1)) continue;
        const long long t = rb_ptr[row] + (long long)rank[w] + __popc(b & ((1u << (cb & 31)) - 1));
        if (at < tiles && t < tiles) {   // (always, unless the pattern changed since its tiles were counted)
            ctile[at] = make_int2(rb, (int)t);
            tile_cb[t] = cb;
        }
        ++at;
    }
}

// One CTA per (pattern, row block), a warp per row: the bits of the tiles.  `masks` begins zeroed.
__global__ void plan_fill_kernel(Csr s, int RB, int words, const unsigned *bitmap, const unsigned *rank, const int *rb_ptr, long long tiles,
                                 unsigned *masks, int *flags)
{
    const int p = blockIdx.x / RB, rb = blockIdx.x % RB;
    const int *rp = s.row_ptr + p * s.rp_stride, *ci = s.col_idx + p * s.nz_stride;
    const unsigned *bm = bitmap + (size_t)blockIdx.x * words, *rk = rank + (size_t)blockIdx.x * words;
    const long long base = rb_ptr[blockIdx.x];
    const int lane = threadIdx.x & 31;
    bool twice = false;
    for (int r = threadIdx.x >> 5; r < kTile && rb * kTile + r < s.M; r += blockDim.x >> 5) {
        int a, e;
        entry_range(rp, s.nz_stride, rb * kTile + r, rb * kTile + r + 1, a, e);
        for (long long i = a; i < e; i += 32) {
            const bool on = i + lane < e;
            const unsigned j = on ? (unsigned)ci[i + lane] : 0xffffffffu;
            if (j < (unsigned)s.K) {
                const unsigned cb = j / kTile, b = bm[cb >> 5];
                const long long t = base + rk[cb >> 5] + __popc(b & ((1u << (cb & 31)) - 1));
                const unsigned m = 1u << (j & 31);
                if (t < tiles && (atomicOr(masks + (t * kTile + r) * 4 + (j >> 5 & 3), m) & m)) twice = true;
            }
        }
    }
    if (twice) atomicOr(flags, kPlanDuplicate);
}

// One CTA of 128 threads per tile, in the order of the column blocks: its transposed bits, and how many each column has.
__global__ void plan_transpose_kernel(int P, int CB, int K, const int *cb_ptr, const int2 *ctile, const uint4 *masks, uint4 *tmasks, int *col_count)
{
    __shared__ unsigned m[kTile][4];
    const long long at = blockIdx.x;
    int lo = 0, hi = P * CB;   // the (pattern, column block) that this tile is of
    while (hi - lo > 1) {
        const int mid = lo + ((hi - lo) >> 1);
        if (cb_ptr[mid] <= at) lo = mid; else hi = mid;
    }
    if (at >= cb_ptr[P * CB]) return;
    const int c = threadIdx.x;
    const uint4 v = masks[(size_t)ctile[at].y * kTile + c];
    m[c][0] = v.x; m[c][1] = v.y; m[c][2] = v.z; m[c][3] = v.w;
    __syncthreads();
    unsigned out[4];
    int n = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        unsigned x = 0;
#pragma unroll 8
        for (int r = 0; r < 32; ++r) x |= (m[w * 32 + r][c >> 5] >> (c & 31) & 1) << r;
        out[w] = x;
        n += __popc(x);
    }
    tmasks[at * kTile + c] = make_uint4(out[0], out[1], out[2], out[3]);
    const int p = lo / CB, j = (lo % CB) * kTile + c;
    if (n && j < K) atomicAdd(col_count + (size_t)p * ((size_t)K + 1) + j, n);
}

// One CTA of 128 threads per (pattern, column block), a thread per column: the rows of each column, ascending.
__global__ void plan_rows_kernel(int CB, int K, const int *cb_ptr, const int2 *ctile, const uint4 *tmasks, const int *col_ptr, long long nz_stride,
                                 int *row_idx)
{
    const int p = blockIdx.x / CB, j = (blockIdx.x % CB) * kTile + threadIdx.x;
    if (j >= K) return;
    long long at = col_ptr[(size_t)p * ((size_t)K + 1) + j];
    int *out = row_idx + p * nz_stride;
    for (long long t = cb_ptr[blockIdx.x]; t < cb_ptr[blockIdx.x + 1]; ++t) {
        const int r0 = ctile[t].x * kTile;
        const uint4 v = tmasks[t * kTile + threadIdx.x];
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            for (unsigned b = w[k]; b; b &= b - 1) {
                if (at < nz_stride) out[at] = r0 + k * 32 + __ffs(b) - 1;
                ++at;
            }
    }
}

}  // namespace attn
}  // namespace b2sp
