// Attention of new tokens over a cache in pages.
//
//   s_j = scale q . k_j;  O = sum_j exp(s_j - m) v_j / l,  l = sum_j exp(s_j - m),  lse = m + log l
//
// over the positions j that a token sees, or those of them in the pages that its list names.
#pragma once
#include "paged.cuh"

namespace b2sp {
namespace paged {

template <typename T> struct AttnArgs {
    Tables t;
    Tokens tok;
    const T *q;
    long long q_ld, q_sh;
    int M, heads, kv_heads, d, page;
    Pages<T> k, v;
    const int *lists;        // [M][kv_heads][keep] or NULL
    int keep;
    float scale;
    T *out;
    long long out_ld, out_sh;
    float *lse;
};

constexpr int kAttnWarps = 4;
// A CTA per token and head, its warps take every fourth position.
template <typename T>
__global__ void __launch_bounds__(kAttnWarps * 32) paged_attention_kernel(const AttnArgs<T> a)
{
    __shared__ float sums[kAttnWarps][256], tops[kAttnWarps], weights[kAttnWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x / a.heads, h = blockIdx.x % a.heads, g = h / (a.heads / a.kv_heads);
    const int seen = seen_of(a.tok, a.t, a.page, i);
    const int *table = a.t.entries + (seen ? row_of(a.tok, i) : 0) * a.t.ld;
    const int *list = a.lists ? a.lists + ((long long)i * a.kv_heads + g) * a.keep : nullptr;
    const int n = seen == 0 ? 0 : list ? a.keep * a.page : seen;
    const T *q = a.q + i * a.q_ld + h * a.q_sh;
    float o[8] = {}, top = -CUDART_INF_F, l = 0.f;
    for (int at = warp; at < n; at += kAttnWarps) {
        int c = at / a.page;
        const int r = at - c * a.page;
        if (list) c = list[c];
        if (c < 0 || c * (long long)a.page + r >= seen) continue;
        const int held = table[c];
        if ((unsigned)held >= (unsigned)a.k.pages) continue;
        const T *k = a.k.row(held, g, r), *v = a.v.row(held, g, r);
        float s = 0.f;
        for (int e = lane; e < a.d; e += 32) s = fmaf(attn::widen(q[e]), attn::widen(k[e]), s);
#pragma unroll
        for (int w = 16; w; w >>= 1) s += __shfl_xor_sync(~0u, s, w);
        s *= a.scale;
        const float to = fmaxf(top, s), ref = to == -CUDART_INF_F ? 0.f : to, fall = expf(top - ref), p = expf(s - ref);
        top = to;
        l = l * fall + p;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = o[j] * fall + (lane + 32 * j < a.d ? p * attn::widen(v[lane + 32 * j]) : 0.f);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[warp][lane + 32 * j] = o[j];
    if (lane == 0) { tops[warp] = top; weights[warp] = l; }
    __syncthreads();
    float high = -CUDART_INF_F;
    for (int w = 0; w < kAttnWarps; ++w) high = fmaxf(high, tops[w]);
    const float ref = high == -CUDART_INF_F ? 0.f : high;
    l = 0.f;
    for (int w = 0; w < kAttnWarps; ++w) l += expf(tops[w] - ref) * weights[w];
    for (int e = threadIdx.x; e < a.d; e += kAttnWarps * 32) {
        float x = 0.f;
        for (int w = 0; w < kAttnWarps; ++w) x += expf(tops[w] - ref) * sums[w][e];
        attn::narrow(l == 0.f ? 0.f : x / l, a.out[i * a.out_ld + h * a.out_sh + e]);
    }
    if (threadIdx.x == 0) a.lse[(long long)i * a.heads + h] = l == 0.f ? -CUDART_INF_F : high + logf(l);
}

}  // namespace paged
}  // namespace b2sp
