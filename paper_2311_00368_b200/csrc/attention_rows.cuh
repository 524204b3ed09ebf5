// Attention over a CSR pattern on the CUDA cores: any pattern, fp32 or bfloat16 operands, any alignment, head widths up to 256.
//
//   forward   s_ij = scale q_i.k_j;  O_i = sum_j exp(s_ij - m_i) v_j / l_i,  l_i = sum_j exp(s_ij - m_i),  lse_i = m_i + log l_i
//   backward  p_ij = exp(s_ij - lse_i);  ds_ij = p_ij (dO_i.v_j - delta_i),  delta_i = dO_i.O_i
//             dQ_i = scale sum_j ds_ij k_j;  dK_j = scale sum_i ds_ij q_i;  dV_j = sum_i p_ij dO_i
//
// A warp takes a row (dK and dV: a column, by the transposed pattern) or one of `splits` equal parts of each, 32 entries at a time.
// Eight lanes form a dot product, the row's own vectors in registers; the sums run with a lane per four output columns (half a warp per
// entry up to 64 columns).  The forward pass keeps a running maximum and sum, so the entries are read once.  Parts of a row are joined
// by a second kernel in a fixed order; nothing depends on the order in which warps run.  All arithmetic is fp32; exponents are taken
// to base 2 (scale log2(e) goes into the factor of the dot product).
//
// What bounds it: the gathers of k_j and v_j from L2 and L1.
#pragma once
#include <math_constants.h>

#include "attention.h"

namespace b2sp {
namespace attn {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Bf16 { unsigned short bits; };
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(Bf16 x) { return __uint_as_float((unsigned)x.bits << 16); }
__device__ __forceinline__ unsigned bf16x2(float lo, float hi)   // round to nearest even
{
    unsigned r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void narrow(float x, float &o) { o = x; }
__device__ __forceinline__ void narrow(float x, Bf16 &o) { o.bits = (unsigned short)bf16x2(x, 0.f); }

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Two fp32 in a register pair, and the instructions that take such pairs.
__device__ __forceinline__ uint64_t two(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(uint64_t x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Elements [c, c + 4) of a row of d elements; V = 4: rows are aligned groups of four.
template <typename T, int V> __device__ __forceinline__ void load4(const T *row, int c, int d, float (&x)[4])
{
    if (V == 4) {
        if (c < d) {
            if constexpr (sizeof(T) == 4) {
                const float4 f = __ldg(reinterpret_cast<const float4 *>(row + c));
                x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
            } else {
                const uint2 u = __ldg(reinterpret_cast<const uint2 *>(row + c));
                x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xffff0000u);
                x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xffff0000u);
            }
        } else {
            x[0] = x[1] = x[2] = x[3] = 0.f;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = c + k < d ? widen(row[c + k]) : 0.f;
    }
}
// The same of partial sums.  They are written by the kernel ahead, which may still run when this one begins: no read-only loads.
__device__ __forceinline__ void load_part(const float *row, int c, int d, float (&x)[4])
{
    const float4 f = c < d ? *reinterpret_cast<const float4 *>(row + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
}
template <typename T, int V> __device__ __forceinline__ void store4(T *row, int c, int d, const float (&x)[4])
{
    if (V == 4) {
        if (c >= d) return;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(row + c) = make_float4(x[0], x[1], x[2], x[3]);
        else *reinterpret_cast<uint2 *>(row + c) = make_uint2(bf16x2(x[0], x[1]), bf16x2(x[2], x[3]));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k < d) narrow(x[k], row[c + k]);
    }
}

enum { kForward = 0, kGradQ = 1, kGradKV = 2 };

template <typename T> struct RowArgs {
    Shape s;
    const int *ptr, *idx;                 // the pattern (kGradKV: the transposed one)
    long long ptr_stride, idx_stride;
    View<const T> q, k, v, dout;
    View<T> out1, out2;                   // O / dQ / dK and dV
    const float2 *stat;                   // backward: (-lse log2(e), -delta) of each row, `stat_stride` rows a problem
    long long stat_stride;
    float *lse;                           // forward; of (b, h, i): lse[b * heads * M + h * lse_head + i * lse_row]
    long long lse_head, lse_row;
    int *status;                          // forward, or NULL: the workspace's status word, set to 0
    int rows, splits;                     // rows: M, or K for kGradKV
    float *part;                          // several parts, or (kGradKV) several query heads per K and V: see part_floats()
    float2 *part_ml;
    int fours_in;                         // rows taken again by the fp32 tile kernels: those of all inputs are aligned groups of four
};
// The partial results of one part of one row: `acc` (kGradKV: two of them), d rounded up to four.
__host__ __device__ constexpr int part_width(int mode, int d) { return ((d + 3) & ~3) * (mode == kGradKV ? 2 : 1); }
// Entries of each part of a row of `len` entries.
__host__ __device__ inline int part_len(int len, int splits) { return splits == 1 ? len : (int)((((long long)len + splits - 1) / splits + 31) & ~31ll); }

// One part of a row: entries [a, e) of idx.  DW: width class of d (64, 128, 256).
template <int MODE, typename T, int V, int DW> struct RowWork {
    static constexpr int KU = DW / 32;               // groups of four that a lane of a dot product holds
    static constexpr int HALVES = DW == 64 ? 2 : 1;  // entries that a sum takes at a time
    static constexpr int AU = DW == 256 ? 2 : 1;     // groups of four output columns per lane
    float acc1[AU][4], acc2[MODE == kGradKV ? AU : 1][4];
    float m, l;

    __device__ __forceinline__ void run(const RowArgs<T> &g, int b, int h, int row, const int *idx, int a, int e)
    {
        const int lane = threadIdx.x & 31, sub = lane & 7, d = g.s.d;
        const int hkv = h / (g.s.heads / g.s.kv_heads);
        const T *own1 = MODE == kGradKV ? g.k.at(b, hkv, row) : g.q.at(b, h, row);
        const T *own2 = MODE == kGradKV ? g.v.at(b, hkv, row) : MODE == kGradQ ? g.dout.at(b, h, row) : nullptr;
        const T *y1 = MODE == kGradKV ? g.q.at(b, h, 0) : g.k.at(b, hkv, 0), *y2 = MODE == kGradKV ? g.dout.at(b, h, 0) : g.v.at(b, hkv, 0);
        const long long ld1 = MODE == kGradKV ? g.q.ld : g.k.ld, ld2 = MODE == kGradKV ? g.dout.ld : g.v.ld;
        const float2 *stat = MODE == kForward ? nullptr : g.stat + ((long long)b * g.s.heads + h) * g.stat_stride;
        const float c2 = g.s.scale * kLog2e;
        float x1[KU][4], x2[MODE == kForward ? 1 : KU][4];
#pragma unroll
        for (int u = 0; u < KU; ++u) {
            load4<T, V>(own1, u * 32 + sub * 4, d, x1[u]);
            if constexpr (MODE != kForward) load4<T, V>(own2, u * 32 + sub * 4, d, x2[u]);
        }
#pragma unroll
        for (int u = 0; u < AU; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                acc1[u][k] = 0.f;
                if constexpr (MODE == kGradKV) acc2[u][k] = 0.f;
            }
        m = -CUDART_INF_F;
        l = 0.f;
        float2 st = make_float2(0.f, 0.f);
        if (MODE == kGradQ) st = stat[row];
        for (long long c = a; c < e; c += 32) {
            const int n = (int)min((long long)32, e - c);
            const int j = lane < n ? idx[c + lane] : 0;
            if (MODE == kGradKV && lane < n) st = stat[j];
            float s = 0.f, dp = 0.f;
#pragma unroll 2
            for (int r = 0; r < 8; ++r) {
                if (r * 4 >= n) break;
                const int at = r * 4 + (lane >> 3), jj = __shfl_sync(~0u, j, at);
                float t1 = 0.f, t2 = 0.f;
                if (at < n) {
                    const T *p1 = y1 + jj * ld1, *p2 = y2 + jj * ld2;
#pragma unroll
                    for (int u = 0; u < KU; ++u) {
                        float y[4];
                        load4<T, V>(p1, u * 32 + sub * 4, d, y);
#pragma unroll
                        for (int k = 0; k < 4; ++k) t1 = fmaf(x1[u][k], y[k], t1);
                        if constexpr (MODE != kForward) {
                            load4<T, V>(p2, u * 32 + sub * 4, d, y);
#pragma unroll
                            for (int k = 0; k < 4; ++k) t2 = fmaf(x2[u][k], y[k], t2);
                        }
                    }
                }
#pragma unroll
                for (int o = 4; o; o >>= 1) {
                    t1 += __shfl_xor_sync(~0u, t1, o);
                    if constexpr (MODE != kForward) t2 += __shfl_xor_sync(~0u, t2, o);
                }
                t1 = __shfl_sync(~0u, t1, (lane & 3) * 8);
                if constexpr (MODE != kForward) t2 = __shfl_sync(~0u, t2, (lane & 3) * 8);
                if ((lane >> 2) == r) { s = t1; dp = t2; }
            }
            float p, w1, w2 = 0.f;   // the weights of the two sums
            if constexpr (MODE == kForward) {
                s = lane < n ? s * c2 : -CUDART_INF_F;
                float top = s;
#pragma unroll
                for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
                top = fmaxf(top, m);
                const float ref = top == -CUDART_INF_F ? 0.f : top;   // logits of -inf only: all weights are 0
                const float fall = exp2f(m - ref);
                p = exp2f(s - ref);
                float sum = p;
#pragma unroll
                for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
                l = fmaf(l, fall, sum);
                m = top;
#pragma unroll
                for (int u = 0; u < AU; ++u)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc1[u][k] *= fall;
                w1 = p;
            } else {
                p = lane < n ? exp2f(fmaf(s, c2, st.x)) : 0.f;
                w1 = lane < n ? p * (dp + st.y) : 0.f;
                w2 = p;
            }
            const int group = HALVES == 2 ? lane >> 4 : 0, col = (HALVES == 2 ? lane & 15 : lane) * 4;
#pragma unroll 4
            for (int i = 0; i < n; i += HALVES) {
                const int at = i + group, jj = __shfl_sync(~0u, j, at & 31);
                const float a1 = __shfl_sync(~0u, w1, at & 31), a2 = MODE == kGradKV ? __shfl_sync(~0u, w2, at & 31) : 0.f;
                if (HALVES == 2 && at >= n) continue;
#pragma unroll
                for (int u = 0; u < AU; ++u) {
                    float y[4];
                    load4<T, V>(MODE == kForward ? y2 + jj * ld2 : y1 + jj * ld1, u * 128 + col, d, y);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc1[u][k] = fmaf(a1, y[k], acc1[u][k]);
                    if constexpr (MODE == kGradKV) {
                        load4<T, V>(y2 + jj * ld2, u * 128 + col, d, y);
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc2[u][k] = fmaf(a2, y[k], acc2[u][k]);
                    }
                }
            }
        }
        if (HALVES == 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                acc1[0][k] += __shfl_xor_sync(~0u, acc1[0][k], 16);
                if constexpr (MODE == kGradKV) acc2[0][k] += __shfl_xor_sync(~0u, acc2[0][k], 16);
            }
        }
    }

    // The finished row.
    __device__ __forceinline__ void finish(const RowArgs<T> &g, int b, int h, int row)
    {
        const int lane = threadIdx.x & 31;
        if (HALVES == 2 && lane >= 16) return;
        const int col = lane * 4, d = g.s.d;
        const int ho = MODE == kGradKV ? h / (g.s.heads / g.s.kv_heads) : h;
        const float f = MODE == kForward ? (l == 0.f ? 0.f : 1.f / l) : g.s.scale;
        T *o1 = g.out1.at(b, ho, row), *o2 = MODE == kGradKV ? g.out2.at(b, ho, row) : nullptr;
#pragma unroll
        for (int u = 0; u < AU; ++u) {
            float x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = acc1[u][k] * f;
            store4<T, V>(o1, u * 128 + col, d, x);
            if constexpr (MODE == kGradKV) store4<T, V>(o2, u * 128 + col, d, acc2[u]);
        }
        if (MODE == kForward && lane == 0)
            g.lse[(long long)b * g.s.heads * g.s.M + h * g.lse_head + row * g.lse_row] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
    }
};

template <int MODE, typename T, int V, int DW>
__global__ void __launch_bounds__(kWarps * 32) attention_row_kernel(const RowArgs<T> g)
{
    const long long unit = blockIdx.x * (long long)kWarps + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (MODE == kForward && g.status && blockIdx.x == 0 && threadIdx.x == 0) *g.status = 0;
    const long long per_problem = (long long)g.rows * g.splits;
    const long long prob = unit / per_problem;
    if (prob >= (long long)g.s.batch * g.s.heads) return;
    const long long in = unit - prob * per_problem, b = (int)(prob / g.s.heads), h = (int)(prob % g.s.heads);
    const int row = (int)(in / g.splits), part = (int)(in % g.splits);
    const int pat = pattern_of(g.s.patterns, g.s.batch, g.s.heads, b, h);
    const int *ptr = g.ptr + pat * g.ptr_stride, *idx = g.idx + pat * g.idx_stride;
    const int first = ptr[row], last = ptr[row + 1], per = part_len(last - first, g.splits);
    const long long a = first + (long long)part * per;
    if (part && a >= last) return;
    RowWork<MODE, T, V, DW> w;
    w.run(g, b, h, row, idx, (int)a, (int)min((long long)last, a + per));
    if (!g.part) {
        w.finish(g, b, h, row);
        return;
    }
    const int width = part_width(MODE, g.s.d), half = part_width(kForward, g.s.d);
    float *o = g.part + unit * width;
    if (w.HALVES == 1 || lane < 16) {
#pragma unroll
        for (int u = 0; u < w.AU; ++u) {
            const int c = u * 128 + lane * 4;
            store4<float, 4>(o, c, half, w.acc1[u]);
            if constexpr (MODE == kGradKV) store4<float, 4>(o + half, c, half, w.acc2[u]);
        }
    }
    if (MODE == kForward && lane == 0) g.part_ml[unit] = make_float2(w.m, w.l);
}

// Joins the parts of a row (kGradKV: of all query heads that share it) in a fixed order.  ROWW warps per row: with many parts (few rows) each
// warp takes every ROWW-th, and the warps' sums are added up in order.
template <int MODE, typename T, int V, int ROWW>
__global__ void __launch_bounds__(kWarps * 32) attention_join_kernel(const RowArgs<T> g)
{
    __shared__ float sums[ROWW == 1 ? 1 : kWarps][MODE == kGradKV ? 2 : 1][256];
    __shared__ float weight[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = g.s.d, group = g.s.heads / g.s.kv_heads;
    const int heads = MODE == kGradKV ? g.s.kv_heads : g.s.heads, mine = ROWW == 1 ? 0 : warp;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long unit = ROWW == 1 ? blockIdx.x * (long long)kWarps + warp : blockIdx.x;
    const long long prob = unit / g.rows;
    if (prob >= (long long)g.s.batch * heads) return;
    const int row = (int)(unit % g.rows), b = (int)(prob / heads), ho = (int)(prob % heads);
    const int width = part_width(MODE, d), half = part_width(kForward, d);
    float acc[MODE == kGradKV ? 2 : 1][2][4] = {};
    float m = -CUDART_INF_F, l = 0.f;
    for (int i = 0; i < (MODE == kGradKV ? group : 1); ++i) {
        const int h = MODE == kGradKV ? ho * group + i : ho;
        const int *ptr = g.ptr + pattern_of(g.s.patterns, g.s.batch, g.s.heads, b, h) * g.ptr_stride;
        const int len = ptr[row + 1] - ptr[row], per = part_len(len, g.splits);
        const int parts = per ? (int)(((long long)len + per - 1) / per) : 1;
        const long long u0 = (((long long)b * g.s.heads + h) * g.rows + row) * g.splits;
        if (MODE == kForward) {
            for (int p = lane; p < parts; p += 32) m = fmaxf(m, g.part_ml[u0 + p].x);
#pragma unroll
            for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
        }
        const float ref = m == -CUDART_INF_F ? 0.f : m;
#pragma unroll 4
        for (int p = mine; p < parts; p += ROWW) {
            float f = 1.f;
            if (MODE == kForward) {
                const float2 ml = g.part_ml[u0 + p];
                f = exp2f(ml.x - ref);
                l = fmaf(ml.y, f, l);
            }
            const float *x = g.part + (u0 + p) * width;
#pragma unroll
            for (int z = 0; z < (MODE == kGradKV ? 2 : 1); ++z)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float y[4];
                    load_part(x + z * half, u * 128 + lane * 4, half, y);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[z][u][k] = fmaf(f, y[k], acc[z][u][k]);
                }
        }
    }
    if (ROWW > 1) {
#pragma unroll
        for (int z = 0; z < (MODE == kGradKV ? 2 : 1); ++z)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                *reinterpret_cast<float4 *>(&sums[warp][z][u * 128 + lane * 4]) = make_float4(acc[z][u][0], acc[z][u][1], acc[z][u][2], acc[z][u][3]);
        if (lane == 0) weight[warp] = l;
        __syncthreads();
        if (warp) return;
        l = 0.f;
#pragma unroll
        for (int z = 0; z < (MODE == kGradKV ? 2 : 1); ++z)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float x = 0.f;
                    for (int w = 0; w < ROWW; ++w) x += sums[w][z][u * 128 + lane * 4 + k];
                    acc[z][u][k] = x;
                }
        for (int w = 0; w < ROWW; ++w) l += weight[w];
    }
    const float f = MODE == kForward ? (l == 0.f ? 0.f : 1.f / l) : g.s.scale;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        float x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = acc[0][u][k] * f;
        store4<T, V>(g.out1.at(b, ho, row), u * 128 + lane * 4, d, x);
        if constexpr (MODE == kGradKV) store4<T, V>(g.out2.at(b, ho, row), u * 128 + lane * 4, d, acc[1][u]);
    }
    if (MODE == kForward && lane == 0) g.lse[(long long)b * g.s.heads * g.s.M + ho * g.lse_head + row * g.lse_row] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
}

// Launches a kernel that begins with griddepcontrol.wait while the one before it still runs.
template <class... KArgs, class... Args>
inline void launch_behind(void (*kern)(KArgs...), unsigned blocks, unsigned threads, cudaStream_t st, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, kern, KArgs(args)...);
}
constexpr int kManyParts = 8;   // from here on four warps join a row
template <int MODE, typename T, int V> inline bool launch_join(const RowArgs<T> &g, cudaStream_t st)
{
    const long long rows = (long long)g.s.batch * (MODE == kGradKV ? g.s.kv_heads : g.s.heads) * g.rows;
    const long long blocks = g.splits >= kManyParts ? rows : (rows + kWarps - 1) / kWarps;
    if (blocks > 0x7fffffff) return false;
    if (g.splits >= kManyParts) launch_behind(attention_join_kernel<MODE, T, V, kWarps>, (unsigned)blocks, kWarps * 32, st, g);
    else launch_behind(attention_join_kernel<MODE, T, V, 1>, (unsigned)blocks, kWarps * 32, st, g);
    return true;
}

// The backward pass's row statistics: (-lse log2(e), -dO_i.O_i), a warp per row, `stat_rows` rows a problem.  A row without entries
// (lse = -inf) and the rows behind the last one get (-inf, 0): exp2(s - inf) = 0, they weigh nothing.
template <typename T, int V>
__global__ void __launch_bounds__(256) attention_stat_kernel(Shape s, View<const T> out, View<const T> dout, const float *lse, int stat_rows, float2 *stat, int *status)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
    const int lane = threadIdx.x & 31;
    const long long unit = blockIdx.x * 8ll + (threadIdx.x >> 5);
    const long long prob = unit / stat_rows;
    if (prob >= (long long)s.batch * s.heads) return;
    const int row = (int)(unit % stat_rows), b = (int)(prob / s.heads), h = (int)(prob % s.heads);
    float sum = 0.f, top = -CUDART_INF_F;
    if (row < s.M) {
        top = lse[prob * s.M + row];
        for (int c = lane * 4; c < s.d; c += 128) {
            float x[4], y[4];
            load4<T, V>(out.at(b, h, row), c, s.d, x);
            load4<T, V>(dout.at(b, h, row), c, s.d, y);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum = fmaf(x[k], y[k], sum);
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane == 0) stat[unit] = top == -CUDART_INF_F ? make_float2(-CUDART_INF_F, 0.f) : make_float2(-top * kLog2e, -sum);
}

}  // namespace attn
}  // namespace b2sp
